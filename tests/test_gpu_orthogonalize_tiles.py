"""GPU tests of pace_orthogonalize on updates whose three products all go in the largest tiles
(test_operators_plans_host.py holds the shapes against the rule); tolerance as in test_gpu_orthogonalize.py."""
import pytest

from tests.test_gpu_orthogonalize import CUBIC, DEV, check, pace, say  # noqa: F401  (pace is the fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
LARGEST = [(1, 4500, 4701), (1, 4609, 9001)]


@pytest.mark.parametrize("batch,rows,cols", LARGEST)
def test_largest_tiles(pace, batch, rows, cols):  # noqa: F811
    say("orthogonalize largest tiles %d x %d x %d" % (batch, rows, cols))
    g = torch.randn(batch, rows, cols, generator=torch.Generator(device=DEV).manual_seed(rows), device=DEV)
    out = check(pace, g, steps=2)
    check(pace, g.transpose(1, 2).contiguous().bfloat16(), steps=1, coefs=CUBIC)
    assert torch.equal(pace.pace_orthogonalize(g, steps=2), out)
