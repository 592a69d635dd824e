"""GPU tests of AdamW's states: what a fresh one holds before its first step, which tensors a step refuses, and what
torch learns of those that it writes."""
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


def test_lists_that_share_memory(pace):
    """In another order, or in part: refused, nothing is written. Neighbours in one buffer are taken."""
    say("adamw of lists that share memory")
    p, g = ([torch.full((n,), 1.5, device=DEV) for n in (300, 300)] for _ in range(2))
    wide, small = pace.adamw_state(p), pace.adamw_state(p, 8)
    flat = torch.full((5000,), 1.5, device=DEV)
    view = lambda *starts: [flat[a: a + 300] for a in starts]
    bytes_of = flat.view(torch.int8)
    for args in ((p, p[::-1], wide), (p, g, dict(wide, exp_avg_sq=wide["exp_avg"][::-1])), (view(0, 1000), view(2000, 1299), wide),
                 (view(0, 1000), g, dict(wide, exp_avg=view(2000, 299))), (p, view(0, 1000), dict(wide, exp_avg_sq=view(1001, 2000))),
                 (view(0, 1000), g, dict(small, exp_avg=[bytes_of[1199: 1499], small["exp_avg"][1]])),
                 (p, g, dict(small, scale=[flat[0:4].view(2, 2), flat[6:10].view(2, 2)], exp_avg=[bytes_of[1000:1300], bytes_of[39:339]])),
                 (view(0, 1000), g, dict(wide, copies=[flat[2000:2150].view(BF16), flat[1299:1449].view(BF16)]))):
        with pytest.raises(ValueError, match="must not overlap each other"):
            pace.pace_adamw(*args)
    with pytest.raises(ValueError, match="must not overlap each other"):
        pace.pace_adamw_unpack(small, out=(view(0, 300), view(1000, 599)))
    torch.cuda.synchronize()
    assert all((t == 1.5).all() for t in p + g + [flat]) and not any(t.any() for t in wide["exp_avg"] + wide["exp_avg_sq"])
    # one behind the other, and one gradient for two parameters
    state = dict(bits=32, scale=None, copies=None, exp_avg=view(600, 900), exp_avg_sq=view(1200, 1500))
    shared = g[:1] * 2
    alone = [t.clone() for t in view(0, 300)], dict(state, **{k: [t.clone() for t in state[k]] for k in ("exp_avg", "exp_avg_sq")})
    pace.pace_adamw(view(0, 300), shared, state)
    pace.pace_adamw(alone[0], [g[0], g[0].clone()], alone[1])
    for a, b in zip(view(0, 300) + state["exp_avg"] + state["exp_avg_sq"], alone[0] + alone[1]["exp_avg"] + alone[1]["exp_avg_sq"]):
        assert torch.equal(a, b)
    # moments of 1.5 beside gradients of 1.5 stay (0.9 and 0.1 of the same), what else there is changes
    assert all((t != 1.5).all() for t in view(0, 300) + state["exp_avg_sq"])
    assert (flat[1800:] == 1.5).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_saved_parameters_and_copies(pace, bits):
    """A pass that saved a parameter or a copy before the step raises, and does not use the new values; one after it runs."""
    say("adamw %d bits, saved parameters" % bits)
    p = [torch.randn(300, device=DEV, requires_grad=True), torch.randn(70, device=DEV, requires_grad=True)]
    x = torch.randn(300, device=DEV, requires_grad=True)
    state = pace.adamw_state(p, bits, BF16)
    step = lambda **kw: pace.pace_adamw(p, [torch.ones_like(t) for t in p], state, **kw)
    for loss in (lambda: sum((t * t).sum() for t in p), lambda: (x * state["copies"][0]).sum()):
        saved = loss()
        step()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            saved.backward()
        saved = loss()
        with pytest.raises(pace.PaceError):
            step(lr=NAN)                             # refused: nothing is written
        for t in p + [x]:
            t.grad = None
        saved.backward()
        assert x.grad is None or torch.equal(x.grad, state["copies"][0].float())
        assert p[0].grad is None or torch.equal(p[0].grad, 2 * p[0])
