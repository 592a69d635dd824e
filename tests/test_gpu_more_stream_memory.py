"""GPU test of the layer norm and AdamW calls on another stream than the current one, without buffers of the caller: what
they allocate is not handed out again on the current stream while their kernels have yet to run."""
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


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


def cases(pace):
    gen = torch.Generator(device=DEV).manual_seed(1)
    f = lambda *shape: torch.randn(*shape, generator=gen, device=DEV)
    x, dy, wide, gw = f(600, 1000), f(600, 1000), f(70, 20000), f(70, 20000)
    stats, wide_stats = pace.pace_layer_norm(x)[1], pace.pace_layer_norm(wide)[1]
    grads = [f(3000000), f(17)]
    state = pace.adamw_state(grads, 8)
    pace.pace_adamw([g.clone() for g in grads], grads, state)
    size = pace.pace_layer_norm_backward_workspace_bytes
    return {
        "layer_norm": (lambda **s: pace.pace_layer_norm(x, **s), x.numel() * 4),
        "layer_norm_backward": (lambda **s: pace.pace_layer_norm_backward(x, stats, dy, **s), size(600, 1000)),
        "layer_norm_backward_wide": (lambda **s: pace.pace_layer_norm_backward(wide, wide_stats, gw, **s), size(70, 20000)),
        "grad_norm": (lambda **s: pace.pace_grad_norm(grads, 1.0, **s), pace.pace_grad_norm_workspace_bytes(2, 3000017)),
        "adamw_unpack": (lambda **s: tuple(t for ts in pace.pace_adamw_unpack(state, **s) for t in ts), 12000000),
        "adamw_state": (lambda **s: tuple(pace.adamw_state(grads, 32, **s)["exp_avg"]), 12000000),
    }


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("name", ["layer_norm", "layer_norm_backward", "layer_norm_backward_wide", "grad_norm", "adamw_unpack", "adamw_state"])
def test_memory_lives_as_long_as_its_kernels(pace, name, handle):
    say("memory of another stream: %s" % name)
    call, size = cases(pace)[name]
    ref = [t.clone() for t in call()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)                # the call's kernels wait behind this
    got = call(stream=side.cuda_stream if handle else side)
    taken = [torch.full((size,), 255, dtype=torch.uint8, device=DEV) for _ in range(4)]
    torch.cuda.current_stream().synchronize()
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, ref))
    assert all(bool((t == 255).all()) for t in taken)
