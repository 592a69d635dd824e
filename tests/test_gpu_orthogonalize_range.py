"""GPU test of the lower end of what pace_orthogonalize holds between its products: elements of X far below the norm.

An update of one large element and, in another row and other columns, small ones x: the norm is the large one, and a
step with coefficients (1.5, -0.5, 0) makes x into 1.5 x, as x's row has next to no length. X is held to 2^-35 of the norm
(half a step of binary16 over 1024) or 2^-11 of x, the product's C to 2^-11, the result to 2^-8: within
2^-34 + (2^-8 + 2^-9) |1.5 x|, without a step within 2^-35 + (2^-8 + 2^-11) |x|."""
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


@pytest.mark.parametrize("rows,cols", [(40, 64), (64, 600), (600, 250), (900, 1000)])
def test_elements_far_below_the_norm(pace, rows, cols):
    """In one workgroup, in launches of two kinds, with the update turned."""
    say("orthogonalize small elements of %d x %d" % (rows, cols))
    g = torch.zeros(1, rows, cols, device=DEV)
    g[0, 0, 0] = 3.0
    x = 3.0 * 1.37 * torch.exp2(-torch.arange(10, 40, device=DEV, dtype=torch.float32))
    g[0, 3, 5:35] = x
    x = (x / 3.0).double()
    for steps, factor, least, rel in ((0, 1.0, 2.0 ** -35, 2.0 ** -8 + 2.0 ** -11), (1, 1.5, 2.0 ** -34, 2.0 ** -8 + 2.0 ** -9)):
        out = pace.pace_orthogonalize(g, steps=steps, coefs=(1.5, -0.5, 0.0)).double()
        assert bool(((out[0, 3, 5:35] - factor * x).abs() <= least + rel * factor * x).all())
        assert abs(float(out[0, 0, 0]) - 1.0) <= 2.0 ** -8
        out[0, 3, 5:35] = 0
        out[0, 0, 0] = 0
        assert not bool(out.any())
