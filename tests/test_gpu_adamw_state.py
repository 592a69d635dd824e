"""GPU tests of AdamW's states: what a fresh one holds before its first step, and what a step tells of the tensors that it writes."""
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
NAN = float("nan")


def say(msg):
    sys.stdout.write("[gpu] %s\n" % msg)
    sys.stdout.flush()


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


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("side", [False, True])
def test_a_first_step_that_is_left_out(pace, bits, dtype, side):
    """The copies are the parameters, also where no step has written them."""
    say("adamw %d bits, first step left out, copies in %s" % (bits, dtype))
    g = torch.Generator(DEV).manual_seed(1)
    params = [torch.randn(n, generator=g, device=DEV) for n in (5000, 1, 0, 300)]
    before = [p.clone() for p in params]
    grads = [torch.randn(p.numel(), generator=g, device=DEV) for p in params]
    stream = torch.cuda.Stream() if side else None
    torch.cuda.synchronize()
    state = pace.adamw_state(params, bits, dtype, stream=stream)
    torch.cuda.synchronize()
    assert all(torch.equal(c, p.to(dtype)) for c, p in zip(state["copies"], params))
    factor = torch.tensor([NAN], device=DEV)
    torch.cuda.synchronize()
    pace.pace_adamw(params, grads, state, step=1, grad_scale=factor, stream=stream)
    torch.cuda.synchronize()
    assert all(torch.equal(p, b) for p, b in zip(params, before))
    assert all(torch.equal(c, p.to(dtype)) for c, p in zip(state["copies"], params))
    pace.pace_adamw(params, grads, state, step=1, stream=stream)
    torch.cuda.synchronize()
    assert all(torch.equal(c, p.to(dtype)) and not torch.equal(p, b) for c, p, b in zip(state["copies"], params, before) if p.numel())
