"""GPU tests of pace_quantize_rows (bit for bit against binary32 steps) and
pace_matmul_i8 (against the exact integer product in binary64).

Tolerance, u = 2^-24: the sum's conversion, the scales' product and the product
with it round once each (3u), the output's type once more (half a unit of its
last place: 2^-24, 2^-9, 2^-11 relative)."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
SUBNORMAL = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
TYPES = [torch.float32, torch.bfloat16, torch.float16]


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


def quantized(x):
    """The definition, in binary32 steps."""
    x = x.float().cpu().numpy()
    with np.errstate(all="ignore"):
        most = np.max(np.abs(x), axis=1)
        bad = ~np.isfinite(x).all(1)
        none = bad | (most < np.float32(2.0 ** -119))
        inv = np.where(none, np.float32(0), np.float32(127) * (np.float32(1) / most)).astype(np.float32)
        q = np.where(none[:, None], 0, np.rint(x * inv[:, None])).astype(np.int8)
        s = np.where(bad, np.float32("nan"), np.where(none, np.float32(0), most / np.float32(127))).astype(np.float32)
    return q, s


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 8), (17, 129), (4, 2048), (300, 1000), (2, 20011)])
def test_quantize(pace, dtype, rows, cols):
    say("quantize %s %d x %d" % (dtype, rows, cols))
    gen = torch.Generator(device=DEV).manual_seed(rows + cols)
    x = (torch.randn(rows, cols, generator=gen, device=DEV) * torch.exp(4 * torch.randn(rows, 1, generator=gen, device=DEV))).to(dtype)
    for view in (x, torch.cat([x.new_full((rows, 3), float("nan")), x, x.new_full((rows, 2), float("inf"))], 1)[:, 3:3 + cols]):
        q, s = pace.pace_quantize_rows(view)
        wq, ws = quantized(x)
        assert np.array_equal(q.cpu().numpy(), wq) and np.array_equal(s.cpu().numpy(), ws)


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_special_rows(pace, dtype):
    say("quantize special rows %s" % dtype)
    x = torch.randn(8, 50, device=DEV).to(dtype)
    x[0] = 0
    x[1] = -0.0
    x[2, 7] = float("nan")
    x[3, 9] = float("-inf")
    x[4] = torch.finfo(dtype).max
    x[5] = torch.finfo(dtype).tiny
    x[6, :] = 0; x[6, 3] = -5.0
    x[7] = torch.arange(50, device=DEV).to(dtype) / 2             # halves: ties to even
    q, s = pace.pace_quantize_rows(x)
    wq, ws = quantized(x)
    assert np.array_equal(q.cpu().numpy(), wq)
    assert np.array_equal(s.cpu().numpy(), ws, equal_nan=True)


def operands(m, n, k, seed, pad=(0, 0), lead=0, extreme=False):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    def ints(rows, extra):
        buf = torch.randint(-128, 128, (lead + rows * (k + extra),), generator=gen, device=DEV, dtype=torch.int8)
        if extreme:
            buf = torch.where(buf >= 0, 127, -128).to(torch.int8)
        return buf[lead:].view(rows, k + extra)[:, :k]
    return (ints(m, pad[0]), torch.rand(m, generator=gen, device=DEV) + 0.1, ints(n, pad[1]),
            torch.rand(n, generator=gen, device=DEV) * 0.01)


def check(pace, a, sa, b, sb, dtype=torch.float32, out=None):
    got = pace.pace_matmul_i8(a, sa, b, sb, out=out, out_dtype=dtype)
    ref = (a.double() @ b.double().t()) * sa.double()[:, None] * sb.double()[None, :]
    err = (got.double() - ref).abs() - ref.abs() * (3 * U + HALF_ULP[got.dtype] * (1 + 3 * U)) - SUBNORMAL[got.dtype]
    assert float(err.max()) <= 0, float(err.max())
    return got


@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 33, 64, 100, 129, 300])
@pytest.mark.parametrize("n,k", [(1, 16), (16, 64), (100, 128), (257, 1024), (1000, 2048), (4096, 144)])
def test_sizes(pace, m, n, k):
    say("i8 product m=%d n=%d k=%d" % (m, n, k))
    check(pace, *operands(m, n, k, m + n + k))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(1, 5000, 4096), (7, 3, 1), (40, 70, 33), (130, 16384, 512), (513, 20001, 272), (2050, 4100, 1040), (256, 256, 8192)])
def test_types(pace, dtype, m, n, k):
    say("i8 product %s m=%d n=%d k=%d" % (dtype, m, n, k))
    check(pace, *operands(m, n, k, k), dtype=dtype)


# Sizes that reach each of the tiles (test_operators_host.py holds them against the rule), with edges off every tile's side.
TILES = [(40, 300, 256), (130, 3001, 1024), (701, 3000, 256), (1100, 1901, 128), (300, 20001, 384), (2001, 2100, 512), (2050, 4101, 1024),
         (4097, 16385, 256), (1021, 70001, 640)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", TILES)
def test_tiles(pace, dtype, m, n, k):
    say("i8 product tiles %s m=%d n=%d k=%d" % (dtype, m, n, k))
    check(pace, *operands(m, n, k, k), dtype=dtype)


# Few tiles of many steps, whose sums are formed in parts (test_operators_host.py holds them against the rule).
PARTS = [(16, 300, 8192), (100, 4097, 6272), (9, 64, 16384), (200, 1001, 8064)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", PARTS)
def test_parts(pace, dtype, m, n, k):
    say("i8 product in parts %s m=%d n=%d k=%d" % (dtype, m, n, k))
    a, sa, b, sb = operands(m, n, k, k, extreme=True)
    ws = torch.full((pace.pace_matmul_i8_workspace_bytes(m, n, k),), 255, dtype=torch.uint8, device=DEV)
    got = pace.pace_matmul_i8(a, sa, b, sb, out_dtype=dtype, workspace=ws)
    assert torch.equal(got, check(pace, a, sa, b, sb, dtype=dtype))


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 5, 7, 8])
@pytest.mark.parametrize("m,n", [(40, 300), (701, 3000), (2001, 2100), (4097, 16385)])
def test_few_steps(pace, m, n, steps):
    """Fewer steps than are held in flight, as many, and more."""
    say("i8 product m=%d n=%d, %d steps" % (m, n, steps))
    check(pace, *operands(m, n, 128 * steps, steps), dtype=torch.bfloat16)


@pytest.mark.parametrize("m", [1, 2, 3, 4, 5, 7, 8, 9])
@pytest.mark.parametrize("n,k,pad,lead", [(1, 1, 0, 0), (7, 130, 0, 0), (700, 4096, 0, 0), (5003, 1000, 0, 0), (9001, 4515, 0, 0), (4097, 2048, 3, 5), (300, 131071, 0, 1)])
def test_few_tokens(pace, m, n, k, pad, lead):
    """One to eight tokens, over weights of every alignment, and the first number beyond them."""
    say("i8 product of %d tokens n=%d k=%d" % (m, n, k))
    a, sa, b, sb = operands(m, n, k, n + k + m, (pad, pad), lead)
    for dtype in TYPES:
        check(pace, a, sa, b, sb, dtype=dtype)


@pytest.mark.parametrize("k", [1, 15, 17, 63, 65, 127, 129, 1000, 1023])
@pytest.mark.parametrize("m,n", [(1, 300), (20, 50), (300, 20000)])
def test_odd_lengths(pace, m, n, k):
    say("i8 product odd k=%d m=%d n=%d" % (k, m, n))
    check(pace, *operands(m, n, k, k))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(30, 900, 259), (300, 20011, 400), (577, 40003, 130), (1000, 25100, 1001)])
def test_tiles_off_alignment(pace, dtype, m, n, k):
    """Each size of tile whose bytes come through registers."""
    say("i8 product off alignment m=%d n=%d k=%d" % (m, n, k))
    check(pace, *operands(m, n, k, m + k), dtype=dtype)


@pytest.mark.parametrize("m,n,k,pad,lead", [(3, 500, 256, (16, 32), 16), (200, 300, 512, (5, 11), 3), (1, 700, 1024, (0, 1), 7),
                                            (300, 17000, 384, (16, 0), 48), (70, 80, 90, (1, 2), 1)])
def test_strides_and_starts(pace, m, n, k, pad, lead):
    """Operands as slices of wider rows, off any alignment; an output inside a wider one, with its surroundings kept."""
    say("i8 product strides m=%d n=%d k=%d" % (m, n, k))
    a, sa, b, sb = operands(m, n, k, 5, pad, lead)
    wide = torch.full((m, n + 9), 7.0, dtype=torch.bfloat16, device=DEV)
    got = check(pace, a, sa, b, sb, out=wide[:, 5:5 + n])
    assert bool((wide[:, :5] == 7).all()) and bool((wide[:, 5 + n:] == 7).all())
    assert torch.equal(got, pace.pace_matmul_i8(a.contiguous(), sa, b.contiguous(), sb))


@pytest.mark.parametrize("m", [1, 20, 200])
def test_longest_sums_are_exact(pace, m):
    """-128 times -128 over the longest rows: the sums stay below 2^31."""
    say("i8 longest sums m=%d" % m)
    k = 131071
    a = torch.full((m, k), -128, dtype=torch.int8, device=DEV)
    b = torch.full((40, k), -128, dtype=torch.int8, device=DEV)
    b[1] = 127
    one = torch.ones(40, device=DEV)
    out = pace.pace_matmul_i8(a, torch.ones(m, device=DEV), b, one, out_dtype=torch.float32)
    assert bool((out[:, 0] == float(np.float32(128 * 128 * k))).all())
    assert bool((out[:, 1] == float(np.float32(-128 * 127 * k))).all())
    check(pace, *operands(m, 40, k, 1, extreme=True))


def test_weights_beyond_32_bits(pace):
    """Weights whose rows lie more than 2^32 bytes from the first."""
    say("i8 product, weights of 4.5 GB")
    n, k = 1100000, 4096
    b = torch.zeros(n, k, dtype=torch.int8, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(2)
    rows = torch.tensor([0, 5, n // 2, n - 2, n - 1], device=DEV)
    b[rows] = torch.randint(-128, 128, (5, k), generator=gen, device=DEV, dtype=torch.int8)
    for m in (1, 30, 140):
        a = torch.randint(-128, 128, (m, k), generator=gen, device=DEV, dtype=torch.int8)
        out = pace.pace_matmul_i8(a, torch.ones(m, device=DEV), b, torch.ones(n, device=DEV), out_dtype=torch.float32)
        ref = (a.double() @ b[rows].double().t()).float()
        assert torch.equal(out[:, rows], ref)
        assert int((out != 0).sum()) == int((ref != 0).sum())


@pytest.mark.parametrize("m", [1, 50, 300])
def test_nan_scales_and_zero_rows(pace, m):
    """A row with a NaN scale is NaN, one with scale 0 is 0, and neither touches other rows."""
    say("i8 scales m=%d" % m)
    a, sa, b, sb = operands(m, 90, 256, 3)
    ref = pace.pace_matmul_i8(a, sa, b, sb)
    sb[4], sb[7] = float("nan"), 0.0
    out = pace.pace_matmul_i8(a, sa, b, sb)
    assert bool(torch.isnan(out[:, 4]).all()) and not bool(out[:, 7].any())
    keep = [i for i in range(90) if i not in (4, 7)]
    assert torch.equal(out[:, keep], ref[:, keep])


@pytest.mark.parametrize("m", [1, 24, 90, 400])
def test_repeats_streams_graph(pace, m):
    say("i8 repeats, streams, graph m=%d" % m)
    x = torch.randn(m, 1024, device=DEV)
    _, _, b, sb = operands(1, 3000, 1024, 6)
    k = pace.matmul_i8_buffers(m, 3000, 1024, torch.bfloat16, DEV)

    def run(stream=None):
        q, s = pace.pace_quantize_rows(x, k["q"], k["scale"], stream=stream)
        pace.pace_matmul_i8(q, s, b, sb, out=k["out"], workspace=k["workspace"], stream=stream)

    run()
    ref = k["out"].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    k["out"].zero_()
    torch.cuda.synchronize()
    run(side)
    torch.cuda.synchronize()
    assert torch.equal(k["out"], ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        for t in k.values():
            t.fill_(3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(k["out"], ref)


def test_rescoring_chain(pace):
    """Hidden states through the quantised head to log-probabilities and the Prefix Forgetting Score: against the same
    chain in binary64 on the quantised values."""
    say("i8 head -> log-probs -> prefix score")
    gen = torch.Generator(device=DEV).manual_seed(9)
    T, K, V = 700, 512, 5000
    hidden = torch.randn(T, K, generator=gen, device=DEV).bfloat16()
    head = 0.1 * torch.randn(V, K, generator=gen, device=DEV)
    hq, hs = pace.pace_quantize_rows(head)
    q, s = pace.pace_quantize_rows(hidden)
    logits = pace.pace_matmul_i8(q, s, hq, hs, out_dtype=torch.float32)
    ids = torch.randint(0, V, (T,), generator=gen, device=DEV, dtype=torch.int32)
    logp = pace.pace_token_logprob(logits, ids)[0]
    z = (q.double() @ hq.double().t()) * s.double()[:, None] * hs.double()[None, :]
    want = torch.log_softmax(z, 1).gather(1, ids.long()[:, None])[:, 0]
    assert float((logp.double() - want).abs().max()) <= 1e-4
    beh = logp + 0.25
    po = torch.tensor([0, 300, 310, T], dtype=torch.int64, device=DEV)
    pre = pace.pace_prefix_score(logp, beh, po)
    assert bool(torch.isnan(pre[1])) and float((pre[[0, 2]] - 0.25).abs().max()) < 1e-6


def test_nothing_to_do(pace):
    say("i8 no rows")
    b, sb = operands(1, 30, 64, 1)[2:]
    assert pace.pace_matmul_i8(torch.empty(0, 64, dtype=torch.int8, device=DEV), torch.empty(0, device=DEV), b, sb).shape == (0, 30)
    assert pace.pace_quantize_rows(torch.empty(0, 64, device=DEV))[0].shape == (0, 64)


def test_refusals(pace):
    say("i8 refusals")
    a, sa, b, sb = operands(4, 6, 64, 1)
    for bad in (lambda: pace.pace_matmul_i8(a.float(), sa, b, sb), lambda: pace.pace_matmul_i8(a, sa, b[:, :32], sb),
                lambda: pace.pace_matmul_i8(a, sa[:3], b, sb), lambda: pace.pace_matmul_i8(a, sa, b, sb.double()),
                lambda: pace.pace_matmul_i8(a.t(), sa, b, sb), lambda: pace.pace_matmul_i8(a.cpu(), sa, b, sb),
                lambda: pace.pace_matmul_i8(a, sa, b, sb, out=torch.empty(4, 5, device=DEV)),
                lambda: pace.pace_matmul_i8(a, sa, b, sb, out_dtype=torch.float64),
                lambda: pace.pace_quantize_rows(a), lambda: pace.pace_quantize_rows(sa),
                lambda: pace.pace_quantize_rows(a.float(), q_out=torch.empty(4, 63, dtype=torch.int8, device=DEV))):
        with pytest.raises(ValueError):
            bad()
    long = torch.zeros(1, 131072, dtype=torch.int8, device=DEV)
    with pytest.raises(pace.PaceError):
        pace.pace_matmul_i8(long, sa[:1], long, sb[:1])
    with pytest.raises(pace.PaceError):
        pace.pace_matmul_i8(a, sa, b, sb, workspace=torch.empty(8, dtype=torch.uint8, device=DEV))


def test_workspace_of_another_place_or_type(pace):
    """A workspace in host memory, or counted in another unit than bytes, is refused before anything runs."""
    a = torch.zeros(3, 64, dtype=torch.int8, device=DEV)
    s = torch.ones(3, device=DEV)
    for bad in (torch.empty(1 << 20, dtype=torch.uint8), torch.empty(1 << 18, dtype=torch.float32, device=DEV)):
        with pytest.raises(ValueError):
            pace.pace_matmul_i8(a, s, a, s, workspace=bad)
