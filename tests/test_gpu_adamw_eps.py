"""GPU test of AdamW with moments in 8 bits at the least eps that it takes, against the formula in 64 bits."""
import math
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


@pytest.fixture(scope="module")
def pace():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import os
    from paper_2609_36830_amd import _lib
    if not os.path.exists(_lib.library_path):
        from paper_2609_36830_amd import build
        build.build()
    import paper_2609_36830_amd as pace
    return pace


@pytest.mark.parametrize("beta2", [0.9, 0.95, 0.999])
def test_second_moments_that_count_as_zero(pace, beta2):
    """Blocks of gradients of one size each, from 1e-30 to 1e-5, then none: some lose their second moments and keep the first."""
    sys.stdout.write("[gpu] adamw 8 bits, least eps, beta2 %g\n" % beta2)
    sys.stdout.flush()
    lr, eps, blocks = 1e-3, 2.0 ** -55 / math.sqrt(1 - beta2) * (1 + 1e-12), 400
    g = torch.Generator(DEV).manual_seed(3)
    sign = torch.randint(0, 2, (blocks, 256), generator=g, device=DEV) * 2.0 - 1.0
    first = (sign * torch.logspace(-30, -5, blocks, dtype=torch.float64, device=DEV)[:, None].float()).view(-1)
    params, grads = [torch.zeros(blocks * 256, device=DEV)], [first.clone()]
    state = pace.adamw_state(params, 8)
    m = v = ref = torch.zeros(blocks * 256, dtype=torch.float64, device=DEV)
    for step in (1, 2, 3):
        pace.pace_adamw(params, grads, state, lr=lr, step=step, betas=(0.9, beta2), eps=eps)
        d = grads[0].double()
        m, v = 0.9 * m + (1 - 0.9) * d, beta2 * v + (1 - beta2) * d * d
        ref = ref - lr / (1 - 0.9 ** step) * m / ((v / (1 - beta2 ** step)).sqrt() + eps)
        # a 256th where v is lost; gradients of one size have codes 127 and 255, which are exact: what is left are 20 roundings of
        # the steps (scales, quotient) and one of the parameter, each step of the same sign
        assert ((params[0].double() - ref).abs() <= (2.0 ** -8 + 2.0 ** -20 + 24 * U) * ref.abs()).all(), step
        if step == 1:
            lost = (state["scale"][0][:, 1] == 0) & (state["scale"][0][:, 0] > 0)
            assert 10 < int(lost.sum()) < blocks - 10
        grads[0].zero_()
    with pytest.raises(pace.PaceError):
        pace.pace_adamw(params, grads, state, lr=lr, step=4, betas=(0.9, beta2), eps=eps / 2)
