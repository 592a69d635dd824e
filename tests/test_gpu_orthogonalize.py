"""GPU tests of pace_orthogonalize against the same steps in binary64.

Tolerance (2-norm of the difference over that of the result), for updates whose
singular values are of one size: a step rounds X, A and C to binary16, each
within 2^-12 root mean square of its own size, and a step passes errors on at
most doubled where singular values stay near the fixed region; over `steps`
steps 6 steps 2^-12. The result's rounding to bfloat16 adds 2^-9."""
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
QUINTIC, CUBIC = (3.4445, -4.7750, 2.0315), (1.5, -0.5, 0.0)


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


def reference(g, steps=5, coefs=QUINTIC, eps=1e-7):
    x = g.double()
    turned = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2) if turned else x
    x = x / (torch.linalg.vector_norm(x, dim=(1, 2), keepdim=True) + eps)
    for _ in range(steps):
        p = x @ x.transpose(1, 2)
        x = coefs[0] * x + (coefs[1] * p + coefs[2] * (p @ p)) @ x
    return x.transpose(1, 2) if turned else x


def check(pace, g, steps=5, coefs=QUINTIC, eps=1e-7, **kw):
    out = pace.pace_orthogonalize(g, steps=steps, coefs=coefs, eps=eps, **kw)
    ref = reference(g if g.dim() == 3 else g[None], steps, coefs, eps)
    got = (out if out.dim() == 3 else out[None]).double()
    rel = torch.linalg.vector_norm(got - ref, dim=(1, 2)) / torch.linalg.vector_norm(ref, dim=(1, 2)).clamp(min=1e-300)
    assert float(rel.max()) <= 6 * steps * 2.0 ** -12 + 2.0 ** -9, float(rel.max())
    return out


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 1), (2, 1, 300), (2, 300, 1), (3, 5, 7), (1, 63, 65), (2, 64, 64), (1, 200, 130),
                                             (4, 128, 513), (1, 1000, 257), (7, 65, 64)])
def test_shapes(pace, dtype, batch, rows, cols):
    say("orthogonalize %s %d x %d x %d" % (dtype, batch, rows, cols))
    g = torch.randn(batch, rows, cols, generator=torch.Generator(device=DEV).manual_seed(rows + cols), device=DEV).to(dtype)
    check(pace, g)
    check(pace, g, steps=3, coefs=CUBIC)


@pytest.mark.parametrize("batch,rows,cols", [(1, 2900, 3001), (1, 4097, 2050), (24, 600, 700), (2, 2048, 2048)])
def test_large_tiles(pace, batch, rows, cols):
    say("orthogonalize %d x %d x %d" % (batch, rows, cols))
    g = torch.randn(batch, rows, cols, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV)
    check(pace, g)


# Shapes whose three products reach each of the tiles (test_operators_host.py holds them against the rule).
TILES = [(1, 2500, 2601), (1, 1000, 3001), (1, 2050, 4097), (2, 1700, 401), (24, 600, 700), (1, 4100, 4200), (3, 1500, 1501)]


@pytest.mark.parametrize("batch,rows,cols", TILES)
def test_tiles(pace, batch, rows, cols):
    say("orthogonalize tiles %d x %d x %d" % (batch, rows, cols))
    g = torch.randn(batch, rows, cols, generator=torch.Generator(device=DEV).manual_seed(rows), device=DEV)
    check(pace, g, steps=2)
    check(pace, g.transpose(1, 2).contiguous().bfloat16(), steps=2)


# Few tiles of many steps in X X^T, whose sums are formed in parts (test_operators_host.py holds them against the rule).
PARTS = [(1, 64, 4096), (2, 128, 2000), (1, 3001, 1000), (1, 8000, 40)]


@pytest.mark.parametrize("batch,rows,cols", PARTS)
def test_parts(pace, batch, rows, cols):
    say("orthogonalize in parts %d x %d x %d" % (batch, rows, cols))
    g = torch.randn(batch, rows, cols, generator=torch.Generator(device=DEV).manual_seed(cols), device=DEV)
    check(pace, g, steps=3)
    b = pace.orthogonalize_buffers(batch, rows, cols, torch.device(DEV))
    b["workspace"].fill_(255)
    first = pace.pace_orthogonalize(g, **b).clone()
    for _ in range(3):
        assert torch.equal(pace.pace_orthogonalize(g, **b), first)


# Updates of few rows, whose C and C X go in one launch (test_operators_host.py holds them against the rule).
SMALL = [(3, 30, 700), (1, 64, 513), (2, 65, 300), (1, 1001, 100), (1, 129, 500), (12, 192, 701), (2, 250, 193), (1, 600, 256), (20, 201, 256)]


@pytest.mark.parametrize("batch,rows,cols", SMALL)
def test_small_steps(pace, batch, rows, cols):
    say("orthogonalize small %d x %d x %d" % (batch, rows, cols))
    g = torch.randn(batch, rows, cols, generator=torch.Generator(device=DEV).manual_seed(rows), device=DEV)
    check(pace, g)
    check(pace, g.half(), steps=1, coefs=CUBIC)
    g[0, 0, 0] = float("nan")                        # its own matrix only
    out = pace.pace_orthogonalize(g)
    assert bool(out[0].isnan().any()) and not bool(out[1:].isnan().any())


# Updates that a workgroup holds whole, up to the largest of both kinds (test_operators_host.py holds them against the rule).
WHOLE = [(3, 30, 200), (1, 1, 512), (2, 64, 449), (2, 512, 64), (1, 64, 512), (2, 65, 127), (5, 128, 256), (1, 256, 127), (2, 193, 65), (300, 20, 33)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("batch,rows,cols", WHOLE)
def test_whole(pace, dtype, batch, rows, cols):
    """Rows apart, off alignment and with other numbers between them; one update's NaN spoils no other."""
    say("orthogonalize whole %s %d x %d x %d" % (dtype, batch, rows, cols))
    gen = torch.Generator(device=DEV).manual_seed(rows + cols)
    room = torch.randn(batch * (rows + 1) * (cols + 5) + 1, generator=gen, device=DEV).to(dtype)
    g = room[1:].view(batch, rows + 1, cols + 5)[:, :rows, 2:cols + 2]
    out = check(pace, g)
    for k in range(0, batch, 2):
        assert torch.equal(pace.pace_orthogonalize(g[k].contiguous()), out[k])
    check(pace, g, steps=1, coefs=CUBIC)
    check(pace, g, steps=8, coefs=CUBIC, eps=0.5)
    if batch > 1:
        g = g.clone()
        g[1, rows - 1, cols - 1] = float("inf")
        bad = pace.pace_orthogonalize(g)
        assert bool(bad[1].isnan().any()) and torch.equal(bad[0], out[0]) and torch.equal(bad[2:], out[2:])


@pytest.mark.parametrize("batch,rows,cols", [(160, 128, 1000), (80, 256, 300), (80, 290, 180)])
def test_alone_as_in_a_batch(pace, batch, rows, cols):
    """A batch that takes C and C X apart gives each update the bits that it has alone, where they go together."""
    say("orthogonalize alone and in a batch %d x %d x %d" % (batch, rows, cols))
    g = torch.randn(batch, rows, cols, generator=torch.Generator(device=DEV).manual_seed(rows), device=DEV)
    out = pace.pace_orthogonalize(g)
    for k in (0, batch // 2, batch - 1):
        assert torch.equal(pace.pace_orthogonalize(g[k]), out[k])


def test_steps_and_coefficients(pace):
    say("orthogonalize steps")
    g = torch.randn(2, 90, 150, generator=torch.Generator(device=DEV).manual_seed(4), device=DEV)
    for steps in (0, 1, 2, 7):
        check(pace, g, steps=steps)
        check(pace, g.transpose(1, 2).contiguous(), steps=steps, coefs=CUBIC)
    check(pace, g, eps=0.5)
    # twenty cubic steps: orthonormal rows to bfloat16's precision
    x = pace.pace_orthogonalize(g, steps=20, coefs=CUBIC).double()
    eye = x @ x.transpose(1, 2)
    assert float((eye - torch.eye(90, device=DEV, dtype=torch.float64)).abs().max()) < 0.02


def test_singular_values_come_together(pace):
    """Singular values from 0.03 to 1 of the largest: five quintic steps bring all into 0.6 .. 1.3."""
    say("orthogonalize singular values")
    gen = torch.Generator(device=DEV).manual_seed(6)
    n = 256
    u, v = (torch.linalg.qr(torch.randn(n, n, generator=gen, device=DEV))[0] for _ in range(2))
    s = torch.linspace(0.2, 1, n, device=DEV)
    x = pace.pace_orthogonalize((u * s) @ v.t())
    got = torch.linalg.svdvals(x.float())
    assert 0.6 < float(got.min()) and float(got.max()) < 1.3


@pytest.mark.parametrize("scale", [1e-30, 1e-3, 1e30, 1e37])
def test_sizes_of_values(pace, scale):
    """The norm's squares leave binary32 at both ends; eps is below the norm throughout."""
    say("orthogonalize values of %g" % scale)
    g = torch.randn(1, 100, 180, generator=torch.Generator(device=DEV).manual_seed(5), device=DEV) * scale
    check(pace, g, eps=1e-36)


def test_special_matrices(pace):
    """Zeros give zeros; NaN and infinities spoil their own matrix only."""
    say("orthogonalize zeros, NaN, infinities")
    g = torch.randn(5, 96, 70, generator=torch.Generator(device=DEV).manual_seed(7), device=DEV)
    ref = pace.pace_orthogonalize(g)
    g[1] = 0
    g[2, 3, 4] = float("nan")
    g[3, 0, 0] = float("inf")
    out = pace.pace_orthogonalize(g)
    assert not bool(out[1].any())
    assert bool(torch.isnan(out[2]).all()) and bool(torch.isnan(out[3]).any())
    assert torch.equal(out[[0, 4]], ref[[0, 4]])


def test_strides(pace):
    """Slices of wider rows and of larger batches, off any alignment; a single matrix without a batch."""
    say("orthogonalize strides")
    buf = torch.full((4, 70, 131), float("nan"), dtype=torch.bfloat16, device=DEV)
    view = buf[::2, 3:63, 1:124]
    view.copy_(torch.randn(2, 60, 123, generator=torch.Generator(device=DEV).manual_seed(8), device=DEV))
    assert torch.equal(pace.pace_orthogonalize(view), pace.pace_orthogonalize(view.contiguous()))
    assert torch.equal(pace.pace_orthogonalize(view[1]), pace.pace_orthogonalize(view.contiguous())[1])


@pytest.mark.parametrize("shape", [(3, 100, 140), (1, 2500, 2600)])
def test_repeats_streams_graph(pace, shape):
    say("orthogonalize repeats, streams, graph %s" % (shape,))
    g = torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(9), device=DEV)
    b = pace.orthogonalize_buffers(*shape, DEV)
    ref = pace.pace_orthogonalize(g, **b).clone()
    b["out"].zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    pace.pace_orthogonalize(g, stream=side, **b)
    torch.cuda.synchronize()
    assert torch.equal(b["out"], ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pace.pace_orthogonalize(g, **b)
    for _ in range(3):
        b["out"].zero_()
        b["workspace"].fill_(255)                    # NaN in every binary16: nothing left by an earlier call is read
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(b["out"], ref)


def test_refusals(pace):
    say("orthogonalize refusals")
    g = torch.randn(2, 30, 40, device=DEV)
    for bad in (lambda: pace.pace_orthogonalize(g.double()), lambda: pace.pace_orthogonalize(g.cpu()), lambda: pace.pace_orthogonalize(g[0, 0]),
                lambda: pace.pace_orthogonalize(g.transpose(1, 2)), lambda: pace.pace_orthogonalize(g, coefs=(1.0, 2.0)),
                lambda: pace.pace_orthogonalize(g, out=torch.empty(2, 30, 41, dtype=torch.bfloat16, device=DEV)),
                lambda: pace.pace_orthogonalize(g, out=torch.empty(2, 30, 40, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: pace.pace_orthogonalize(g, steps=-1), lambda: pace.pace_orthogonalize(g, steps=101), lambda: pace.pace_orthogonalize(g, eps=0.0),
                lambda: pace.pace_orthogonalize(g, coefs=(float("nan"), 0, 0)),
                lambda: pace.pace_orthogonalize(g, workspace=torch.empty(64, dtype=torch.uint8, device=DEV)),
                lambda: pace.pace_orthogonalize(g[0][:, :0])):
        with pytest.raises(pace.PaceError):
            bad()


def test_workspace_of_another_place_or_type(pace):
    """A workspace in host memory, or counted in another unit than bytes, is refused before anything runs."""
    for bad in (torch.empty(1 << 20, dtype=torch.uint8), torch.empty(1 << 18, dtype=torch.float32, device=DEV)):
        with pytest.raises(ValueError):
            pace.pace_orthogonalize(torch.zeros(8, 8, device=DEV), workspace=bad)
