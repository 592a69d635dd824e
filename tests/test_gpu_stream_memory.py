"""GPU test of calls on another stream than the current one, without buffers of the caller: what the call allocates is
not handed out again on the current stream while the call's kernels have yet to run."""
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
    z, ids = f(6, 60001).bfloat16(), torch.randint(0, 60001, (6,), generator=gen, device=DEV, dtype=torch.int32)
    off = torch.tensor([0, 70000, 70001, 200003], device=DEV)
    new, beh, adv = f(200003) - 1.0, f(200003) - 1.0, f(3)
    i8 = lambda *shape: torch.randint(-128, 128, shape, generator=gen, device=DEV, dtype=torch.int8)
    a, b, sa, sb = i8(16, 8192), i8(300, 8192), torch.rand(16, device=DEV), torch.rand(300, device=DEV)
    update = f(1, 300, 2000)
    score = torch.rand(9000, generator=gen, device=DEV, dtype=torch.float64)
    stats = pace.pace_token_logprob(z, ids)[2]
    return {
        "token_logprob": (lambda **s: pace.pace_token_logprob(z, ids, 1.0, 20, **s), pace.pace_token_logprob_workspace_bytes(6, 60001, 20)),
        "backward": (lambda **s: (pace.pace_token_logprob_backward(z, ids, stats, adv.repeat(2), **s),), z.numel() * 2),
        "policy_loss": (lambda **s: pace.pace_policy_loss(new, beh, off, adv, **s), pace.pace_policy_loss_workspace_bytes(3, 200003)),
        "matmul_i8": (lambda **s: (pace.pace_matmul_i8(a, sa, b, sb, **s),), pace.pace_matmul_i8_workspace_bytes(16, 300, 8192)),
        "orthogonalize": (lambda **s: (pace.pace_orthogonalize(update, **s),), pace.pace_orthogonalize_workspace_bytes(1, 300, 2000)),
        "select": (lambda **s: pace.pace_select(score, 1000, **s), pace.pace_workspace_bytes(pace.WS_SELECT, 9000, 0)),
    }


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("name", ["token_logprob", "backward", "policy_loss", "matmul_i8", "orthogonalize", "select"])
def test_workspace_lives_as_long_as_its_kernels(pace, name, handle):
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
