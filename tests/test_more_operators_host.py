"""CPU tests of the host checks of the layer norm, the gradients' norm and AdamW (every refusal returns before any launch),
and of their rules on sizes (csrc/rules.hpp, compiled for the host)."""
import ctypes
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x100000   # aligned, never dereferenced
SOURCE = """
#include "%s"
using namespace pace;
extern "C" {
int64_t lanes(int64_t cols) { return layer_norm_lanes(cols); }
int64_t rows_of(int64_t lanes) { return layer_norm_backward_rows((int)lanes); }
int64_t parts(int64_t rows, int64_t cols) { return layer_norm_backward_parts(rows, cols); }
int64_t floats(int64_t rows, int64_t cols) { return parts(rows, cols) * 2 * ((cols + 3) / 4 * 4); }
int64_t floats_most(int64_t rows, int64_t cols) { return layer_norm_part_floats_most(rows, cols); }
int64_t chunk(int64_t n) { return grad_norm_chunk(n); }
int64_t slots_most(int64_t k, int64_t n) { return grad_norm_slots_most(k, n); }
int64_t turns(int64_t n) { return adamw_turns(n); }
// Tables of at most 5 tensors and `most` workgroups: how many, or a negative number where a tensor that is taken (every
// number but 3 k + 1) is not in one of them in order, with the workgroups that its elements need.
int64_t tables(int64_t n, const int64_t *sizes, int64_t per, int64_t most, int64_t fail_at) {
    int64_t next = 0, count = 0, wrong = 0;
    const int e = by_tables<int, int64_t, 5>(n, sizes, per, most, [&](int64_t i, int64_t &to) { to = i; return i %% 3 != 1; },
        [&](const Table<int64_t, 5> &t, int64_t blocks) {
            int64_t at = 0;
            if (blocks < 1 || blocks > most) wrong = 1;
            for (int k = 0; k < 5; ++k) {
                if (t.first[k] == UINT32_MAX) {
                    if (k == 0) wrong = 2;
                    continue;
                }
                while (next < n && (sizes[next] == 0 || next %% 3 == 1)) ++next;
                if (t.entry[k] != next || t.first[k] != at || (k > 0 && t.first[k - 1] == UINT32_MAX)) wrong = 3;
                at += (sizes[next++] + per - 1) / per;
            }
            if (at != blocks) wrong = 4;
            return count++ == fail_at ? 7 : 0;
        });
    while (next < n && (sizes[next] == 0 || next %% 3 == 1)) ++next;
    if (e != (fail_at >= 0 && count > fail_at ? 7 : 0) || (e == 0 && next != n)) wrong = 5;
    return wrong ? -wrong : count;
}
}
""" % os.path.join(ROOT, "paper_2609_36830_amd", "csrc", "rules.hpp")


@pytest.fixture(scope="module")
def R(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "r.cpp").write_text(SOURCE)
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", str(d / "r.cpp"), "-o", str(d / "r.so")])
    lib = ctypes.CDLL(str(d / "r.so"))
    for name, n in (("lanes", 1), ("rows_of", 1), ("parts", 2), ("floats", 2), ("floats_most", 2), ("chunk", 1), ("slots_most", 2), ("turns", 1)):
        getattr(lib, name).restype, getattr(lib, name).argtypes = ctypes.c_int64, [ctypes.c_int64] * n
    lib.tables.restype, lib.tables.argtypes = ctypes.c_int64, [ctypes.c_int64, ctypes.c_void_p] + [ctypes.c_int64] * 3
    return lib


@pytest.fixture(scope="module")
def L():
    from paper_2609_36830_amd import _lib
    if not os.path.exists(_lib.library_path):
        from paper_2609_36830_amd import build
        build.build()
    return _lib.lib()


def log_int(rng, most):
    return max(1, int(2 ** rng.uniform(0, most.bit_length() - 1)))


def test_layer_norm_host_argument_errors(L):
    def call(x=FAKE, dt=1, n=4, k=100, st=100, w=FAKE, b=FAKE, wt=0, eps=1e-5, out=2 * FAKE, ost=100, stats=FAKE):
        return L.pace_layer_norm(x, dt, n, k, st, w, b, wt, eps, out, ost, stats, None)

    for kw in (dict(x=None), dict(out=None), dict(x=FAKE + 1), dict(out=FAKE + 1), dict(dt=3), dict(dt=-1), dict(wt=2), dict(wt=-1), dict(wt=3),
               dict(dt=0, wt=1), dict(n=-1), dict(n=2 ** 31), dict(k=0), dict(k=2 ** 24 + 1, st=2 ** 25, ost=2 ** 25), dict(st=99), dict(ost=99),
               dict(n=2 ** 31 - 2, st=2 ** 40), dict(w=FAKE + 2), dict(b=FAKE + 2), dict(stats=FAKE + 2), dict(eps=0.0), dict(eps=-1.0),
               dict(eps=1e-31), dict(out=FAKE), dict(eps=float("inf")), dict(eps=float("nan"))):
        assert call(**kw) == -1, kw


def test_layer_norm_backward_host_argument_errors(L):
    def call(x=FAKE, dt=1, n=4, k=100, st=100, w=FAKE, wt=1, stats=FAKE, dy=2 * FAKE, dyst=100, dx=3 * FAKE, dxst=100, dw=FAKE, db=FAKE,
             ws=FAKE, wsb=1 << 30):
        return L.pace_layer_norm_backward(x, dt, n, k, st, w, wt, stats, dy, dyst, dx, dxst, dw, db, ws, wsb, None)

    for kw in (dict(x=None), dict(dy=None), dict(dx=None), dict(stats=None), dict(dt=5), dict(wt=2), dict(n=-1), dict(k=0), dict(st=99),
               dict(dyst=99), dict(dxst=99), dict(dx=2 * FAKE, dxst=101), dict(dx=FAKE), dict(w=FAKE + 1), dict(stats=FAKE + 2),
               dict(dw=FAKE + 2), dict(db=FAKE + 1)):
        assert call(**kw) == -1, kw
    for kw in (dict(ws=None), dict(ws=FAKE + 128), dict(wsb=256), dict(dw=None, wsb=256), dict(db=None, wsb=256)):
        assert call(**kw) == -2, kw
    out = ctypes.c_size_t()
    for n, k in ((-1, 5), (2 ** 31, 5), (5, 0), (5, 2 ** 24 + 1)):
        assert L.pace_layer_norm_backward_workspace_bytes(n, k, ctypes.byref(out)) == -1
    assert L.pace_layer_norm_backward_workspace_bytes(5, 5, None) == -1


def arrays(n, values):
    """[host] arrays of n tensors: pointers, types, sizes."""
    return {name: (kind * n)(*([v] * n if not isinstance(v, (list, tuple)) else v)) for name, kind, v in values}


P, I32, I64, FL = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


def test_grad_norm_host_argument_errors(L):
    def call(n=2, g=(FAKE, FAKE), dt=(0, 1), sizes=(5, 7), most=1.0, norm=FAKE, factor=FAKE, ws=FAKE, wsb=1 << 20, none=()):
        a = arrays(2, (("g", P, g), ("dt", I32, dt), ("sizes", I64, sizes)))
        a.update((k, None) for k in none)
        return L.pace_grad_norm(n, a["g"], a["dt"], a["sizes"], most, norm, factor, ws, wsb, None)

    for kw in (dict(n=-1), dict(g=(FAKE, None)), dict(g=(FAKE + 2, FAKE)), dict(g=(FAKE, FAKE + 1)), dict(dt=(0, 3)), dict(dt=(-1, 0)),
               dict(sizes=(5, -1)), dict(sizes=(5, 2 ** 35 + 1)), dict(most=-1.0), dict(most=float("nan")), dict(norm=None, factor=None),
               dict(norm=FAKE + 2), dict(none=("g",)), dict(none=("dt",)), dict(none=("sizes",))):
        assert call(**kw) == -1, kw
    for kw in (dict(ws=None), dict(ws=FAKE + 8), dict(wsb=100), dict(sizes=(2 ** 30, 2 ** 30), wsb=1 << 15)):
        assert call(**kw) == -2, kw


def test_adamw_host_argument_errors(L):
    from paper_2609_36830_amd._lib import AdamwParams

    def call(n=2, bits=8, none=(), hyper=(1e-3, 0.9, 0.99, 1e-8, 1), factor=FAKE, schedule=None, **kw):
        a = arrays(2, [(k, t, kw.pop(k, d)) for k, t, d in (
            ("sizes", I64, (5, 300)), ("p", P, FAKE), ("pt", I32, 0), ("g", P, FAKE), ("gt", I32, (1, 2)), ("m", P, FAKE), ("v", P, FAKE),
            ("scale", P, FAKE), ("copy", P, (FAKE, None)), ("ct", I32, (1, 7)), ("decay", FL, 0.1))])
        assert not kw
        a.update((k, None) for k in none)
        h = ctypes.byref(AdamwParams(*hyper)) if hyper is not None else None
        return L.pace_adamw(n, a["sizes"], a["p"], a["pt"], a["g"], a["gt"], bits, a["m"], a["v"], a["scale"], a["copy"], a["ct"], a["decay"],
                            h, factor, schedule, None)

    nan, inf = float("nan"), float("inf")
    for kw in (dict(n=-1), dict(bits=16), dict(bits=0), dict(sizes=(5, -300)), dict(sizes=(5, 2 ** 35 + 1)), dict(p=(FAKE, None)), dict(p=FAKE + 2),
               dict(pt=(0, 3)), dict(g=(None, FAKE)), dict(g=(FAKE + 1, FAKE)), dict(gt=(-1, 0)), dict(m=(FAKE, None)), dict(v=(FAKE, None)),
               dict(bits=32, m=FAKE + 1), dict(bits=32, v=FAKE + 2), dict(scale=(FAKE, None)), dict(scale=FAKE + 2), dict(copy=(FAKE + 1, None)),
               dict(ct=(0, 0)), dict(ct=(3, 0)), dict(decay=(0.1, -0.1)), dict(decay=(0.1, nan)), dict(decay=(inf, 0.0)), dict(hyper=None),
               dict(hyper=(nan, 0.9, 0.99, 1e-8, 1)), dict(hyper=(inf, 0.9, 0.99, 1e-8, 1)), dict(hyper=(1e-3, 1.0, 0.99, 1e-8, 1)),
               dict(hyper=(1e-3, 0.9, nan, 1e-8, 1)), dict(hyper=(1e-3, -0.1, 0.99, 1e-8, 1)), dict(hyper=(1e-3, 0.9, 0.99, 0.0, 1)),
               dict(hyper=(1e-3, 0.9, 0.99, 1e31, 1)), dict(hyper=(1e-3, 0.9, 0.99, 1e-8, 0)), dict(factor=FAKE + 2), dict(schedule=FAKE + 4),
               *(dict(none=(k,)) for k in ("sizes", "p", "pt", "g", "gt", "m", "v", "scale", "ct"))):
        assert call(**kw) == -1, kw
    # a schedule stands in for lr and step; nothing to do is no error and no launch
    assert call(n=0, none=("sizes", "p", "pt", "g", "gt", "m", "v", "scale", "copy", "ct", "decay")) == 0
    assert call(sizes=(0, 0), p=None, g=None, m=None, v=None, scale=None, schedule=FAKE, hyper=(nan, 0.9, 0.99, 1e-8, 0)) == 0


def test_adamw_unpack_host_argument_errors(L):
    def call(n=2, none=(), **kw):
        a = arrays(2, [(k, t, kw.pop(k, d)) for k, t, d in (("sizes", I64, (5, 300)), ("m", P, FAKE), ("v", P, FAKE), ("scale", P, FAKE),
                                                            ("mo", P, FAKE), ("vo", P, FAKE))])
        a.update((k, None) for k in none)
        return L.pace_adamw_unpack(n, a["sizes"], a["m"], a["v"], a["scale"], a["mo"], a["vo"], None)

    for kw in (dict(n=-1), dict(sizes=(5, -1)), dict(m=(FAKE, None)), dict(v=(None, FAKE)), dict(scale=FAKE + 2), dict(mo=(FAKE, None)),
               dict(vo=FAKE + 2), dict(none=("mo", "vo")), dict(none=("m",)), dict(none=("v",)), dict(none=("scale",)), dict(none=("sizes",))):
        assert call(**kw) == -1, kw
    assert call(sizes=(0, 0)) == 0


def test_layer_norm_lanes_and_parts(R):
    """A row fits its lanes; no chain of rows is longer than 1024, no part without a workgroup that a grid can hold."""
    rng = random.Random(1)
    for cols in list(range(1, 2000)) + [4096, 4097, 8192, 16384]:
        n = R.lanes(cols)
        assert n * 16 >= cols and (n == 8 or n * 8 < cols) and n in (8, 16, 32, 64, 128, 256, 512, 1024)
    for _ in range(5000):
        rows, cols = log_int(rng, 2 ** 31 - 2), log_int(rng, 2 ** 24)
        p = R.parts(rows, cols)
        assert 1 <= p <= rows and p <= 2 ** 26
        if cols <= 16384:
            assert p * R.rows_of(R.lanes(cols)) * 1024 >= rows
        else:
            assert p <= 65535
    assert R.parts(0, 100) == R.parts(0, 20000) == 0


def test_layer_norm_workspace_of_every_smaller_problem(R):
    rng = random.Random(2)
    for _ in range(20000):
        rows, cols = log_int(rng, 2 ** 24), log_int(rng, 2 ** 16)
        r, c = rng.randint(0, rows), rng.randint(1, cols)
        assert R.floats(r, c) <= R.floats_most(rows, cols)
        assert R.floats_most(r, c) <= R.floats_most(rows, cols)


def test_grad_norm_sums_of_every_smaller_call(R):
    rng = random.Random(3)
    for _ in range(5000):
        most, total = log_int(rng, 2000), log_int(rng, 2 ** 36)
        k, n = rng.randint(1, most), rng.randint(0, total)
        cuts = sorted(rng.randint(0, n) for _ in range(k - 1))
        sizes = [b - a for a, b in zip([0] + cuts, cuts + [n])]
        chunk = R.chunk(n)
        assert sum(-(-s // chunk) for s in sizes) <= R.slots_most(most, total)
        assert R.slots_most(k, n) <= R.slots_most(most, total)


def test_tables_hold_every_tensor_once(R):
    rng = random.Random(4)
    for _ in range(3000):
        most, per, n = rng.choice([4, 9, 1000]), rng.choice([1, 7, 4096]), rng.randint(0, 40)
        sizes = [rng.choice([0, 1, per, per + 1, rng.randint(0, most * per), most * per]) for _ in range(n)]
        a = (ctypes.c_int64 * max(n, 1))(*sizes)
        count = R.tables(n, a, per, most, -1)
        taken = [s for k, s in enumerate(sizes) if s and k % 3 != 1]
        assert -(-len(taken) // 5) <= count <= len(taken)
        if count > 1:                                # an error ends it
            assert R.tables(n, a, per, most, count - 2) == count - 1


def test_gpu_tests_reach_every_form(R):
    """Rows of every number of lanes, whole and ragged, and wider ones; steps of one round a workgroup and of two."""
    from tests.test_gpu_adamw import SIZES
    from tests.test_gpu_layer_norm import SHAPES
    for vec in (4, 8):
        forms = {(R.lanes(c) if c <= 16384 else 0, c % vec == 0) for _, c in SHAPES}
        assert {f for f, _ in forms} == {0, 8, 16, 32, 64, 128, 256, 512, 1024}
        assert forms >= {(n, whole) for n in (8, 16, 32, 64, 128, 256, 512, 1024) for whole in (True, False)}, forms
        # rows beyond one turn of the forward pass's workgroups, and of the backward pass's
        assert any(r > R.parts(r, c) * R.rows_of(R.lanes(c)) for r, c in SHAPES if c <= 16384)
    assert {R.turns(sum(s)) for s in SIZES} == {1, 2}


def test_lists_are_refused_before_any_call(L):
    """What is no contiguous device tensor of the right type never reaches the library."""
    import torch
    import paper_2609_36830_amd as pace
    x = torch.zeros(6)
    for bad in ([x], [3], [None], (x.numpy(),), [x.to_sparse()], [torch.zeros(6, device="meta")], [], 7):
        with pytest.raises((ValueError, TypeError)):
            pace.pace_grad_norm(bad)
        with pytest.raises((ValueError, TypeError)):
            pace.adamw_state(bad)
    read = pace._lib.lists().read
    with pytest.raises(ValueError, match=r"grads must hold 2 tensors"):
        read([x], "grads", 7, 0, False, b"\0" * 16, 0)
    with pytest.raises(ValueError, match=r"grads\[0\] must be a contiguous device tensor of float32 or float16"):
        read([x], "grads", 5, 0, False, b"\0" * 8, 0)
    with pytest.raises(ValueError, match="sizes must be bytes"):
        read([], "grads", 7, 0, False, 3, 0)
    assert read([], "grads", 7, 0, True, b"", 0) == (0, 0, b"", b"", b"", 0)
    m = pace._lib.lists()
    for bad in (x, 3, None, torch.zeros(2, 3), torch.zeros(2, 3, device="meta"), torch.zeros(2, 3).to_sparse()):
        with pytest.raises(ValueError):
            m.matrix(bad, "x", 7, -1, -1, -1)
        with pytest.raises(ValueError, match="x must be a"):
            m.vector(bad, "x", 7, -1, -1)
    with pytest.raises(ValueError, match="x must be a device tensor of float32 or bfloat16 or float16"):
        pace.pace_layer_norm(torch.zeros(2, 3))
    with pytest.raises(ValueError):
        pace.adamw_state([x], bits=8)
    with pytest.raises(ValueError, match="8 bits"):
        pace.pace_adamw_unpack(dict(bits=32))


def test_the_same_tensor_in_two_lists(L):
    import array
    import paper_2609_36830_amd as pace
    apart = pace._lib.lists().apart
    of = lambda *p: array.array("Q", p).tobytes()
    assert apart(("a", "b", "c"), (of(1, 2, 0), None, of(2, 1, 0))) is None       # empty tensors have no place
    assert apart((), ()) is None and apart(("a", "b"), (b"", b"")) is None
    with pytest.raises(ValueError, match="a and c must not overlap each other"):
        apart(("a", "b", "c"), (of(1, 2, 5), of(3, 4, 6), of(7, 8, 5)))
    for bad in ((("a",), ()), (("a", "b"), (of(1), of(1, 2))), ((1, "b"), (of(1), of(2))), (("a", "b"), (3, of(2))), (["a"], (of(1),)), (3, 4)):
        with pytest.raises((ValueError, TypeError)):
            apart(*bad)
