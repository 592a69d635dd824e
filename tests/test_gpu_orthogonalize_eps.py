"""GPU test of pace_orthogonalize with an eps near 0: zero updates give zeros, the smallest updates their direction."""
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


@pytest.mark.parametrize("steps", [0, 1, 5])
@pytest.mark.parametrize("eps", [1e-7, 1e-300, 1e-306, 5e-324])
@pytest.mark.parametrize("rows,cols", [(30, 50), (200, 130), (64, 600)])
def test_small_eps(pace, rows, cols, eps, steps):
    """In one workgroup, in launches of two kinds, and without steps."""
    say("orthogonalize %d x %d, eps %g, %d steps" % (rows, cols, eps, steps))
    g = torch.randn(3, rows, cols, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    g[1] = 0
    ref = pace.pace_orthogonalize(g, steps=steps, eps=1e-30)
    out = pace.pace_orthogonalize(g, steps=steps, eps=eps)
    assert not bool(out[1].any())
    if eps < 1e-30:                                  # the factor is the same binary64 number
        assert torch.equal(out, ref)
        least = torch.zeros_like(g)
        least[0, 0, 0] = 1e-45                       # the least binary32 number
        got = pace.pace_orthogonalize(least, steps=0, eps=eps)
        assert float(got[0, 0, 0]) == 1.0 and not bool(got[1:].any())
