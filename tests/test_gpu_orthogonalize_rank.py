"""GPU test of pace_orthogonalize on updates of low rank, whose missing directions hold what rounding leaves there.

Tolerance. A step rounds X, A and C to binary16, each error random and at most 2^-12 root mean square of its matrix, and
what falls into a direction without a singular value grows by the first coefficient a step, as X itself does while its
values are small. From |X| = 1 the 3 roundings of each of `steps` steps end, added as squares, at
sqrt(3 steps) 2^-12 a^steps; the result has k singular values of 0.7 to 1.2, a 2-norm of 0.7 sqrt(k) at least. With
the error of the other directions (test_gpu_orthogonalize.py's) the sum of both."""
import math

import pytest

from tests.test_gpu_orthogonalize import DEV, QUINTIC, pace, reference, say  # noqa: F401  (pace is the fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols,k", [(16, 16, 2), (64, 512, 8), (256, 256, 32), (200, 1000, 1), (1000, 900, 100), (2000, 2600, 300)])
def test_low_rank(pace, rows, cols, k):  # noqa: F811
    say("orthogonalize %d x %d of rank %d" % (rows, cols, k))
    gen = torch.Generator(device=DEV).manual_seed(rows)
    u, v = (torch.linalg.qr(torch.randn(n, k, generator=gen, device=DEV))[0] for n in (rows, cols))
    g = ((u * torch.linspace(0.5, 1, k, device=DEV)) @ v.t())[None]
    steps = 5
    ref, out = reference(g, steps), pace.pace_orthogonalize(g, steps=steps).double()
    rel = float(torch.linalg.vector_norm(out - ref) / torch.linalg.vector_norm(ref))
    assert rel <= math.sqrt(3 * steps) * 2.0 ** -12 * QUINTIC[0] ** steps / (0.7 * math.sqrt(k)) + 6 * steps * 2.0 ** -12 + 2.0 ** -9, rel
    # in its own directions it is the reference as closely as any update
    own = u.double().t() @ (out - ref)[0] @ v.double()
    assert float(own.norm() / torch.linalg.vector_norm(ref)) <= 6 * steps * 2.0 ** -12 + 2.0 ** -9
