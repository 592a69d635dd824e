"""CPU tests of the host checks of the operators around the filter step: every
refusal returns before any launch, so no GPU is needed."""
import os

import pytest

FAKE = 0x100000   # aligned, never dereferenced


@pytest.fixture(scope="module")
def L():
    from paper_2609_36830_amd import _lib
    if not os.path.exists(_lib.library_path):
        from paper_2609_36830_amd import build
        build.build()
    return _lib.lib()


def test_token_logprob_host_argument_errors(L):
    def call(z=FAKE, dt=0, n=4, v=100, st=100, ids=FAKE, t=1.0, k=0, lp=FAKE, ti=FAKE, tl=FAKE, ws=FAKE, wsb=1 << 30):
        return L.pace_token_logprob(z, dt, n, v, st, ids, t, k, lp, FAKE, FAKE, ti, tl, ws, wsb, None)

    for kw in (dict(z=None), dict(z=FAKE + 2), dict(dt=3), dict(dt=-1), dict(n=-1), dict(v=0), dict(v=2 ** 31), dict(st=99),
               dict(n=2 ** 31 - 2, st=2 ** 40), dict(ids=None), dict(ids=FAKE + 2), dict(t=0.0), dict(t=-1.0), dict(t=1e-7),
               dict(t=float("inf")), dict(t=float("nan")), dict(k=-1), dict(k=65), dict(v=10, st=10, k=11), dict(lp=None),
               dict(k=3, ti=None), dict(k=3, tl=None), dict(lp=FAKE + 1)):
        assert call(**kw) == -1, kw
    for kw in (dict(ws=None), dict(ws=FAKE + 64), dict(wsb=64), dict(n=2, v=150000, st=150000, k=20, wsb=4096)):
        assert call(**kw) == -2, kw
    assert call(dt=1, z=FAKE + 2, wsb=0) == -2          # two-byte elements need two-byte alignment only


def test_token_logprob_backward_host_argument_errors(L):
    def call(z=FAKE, dt=0, n=4, v=100, st=100, ids=FAKE, t=1.0, stats=FAKE, ent=FAKE, g=FAKE, ge=None, out=FAKE * 2, ost=100):
        return L.pace_token_logprob_backward(z, dt, n, v, st, ids, t, stats, ent, g, ge, out, ost, None)

    for kw in (dict(z=None), dict(out=None), dict(ost=99), dict(dt=4), dict(t=0.0), dict(stats=None), dict(g=None), dict(ids=None),
               dict(ent=None, ge=FAKE), dict(out=FAKE, ost=101), dict(g=FAKE + 2), dict(n=-1)):
        assert call(**kw) == -1, kw


def test_token_logprob_workspace(L):
    import paper_2609_36830_amd as pace
    assert pace.pace_token_logprob_workspace_bytes(0, 10) >= 256
    assert pace.pace_token_logprob_workspace_bytes(10 ** 6, 150000, 64) < 1 << 20      # whole rows: nothing to join
    for bad in ((-1, 10, 0), (1, 0, 0), (1, 10, 65)):
        with pytest.raises(pace.PaceError):
            pace.pace_token_logprob_workspace_bytes(*bad)


def test_policy_loss_host_argument_errors(L):
    def call(new=FAKE, beh=FAKE, tags=None, off=FAKE, n=4, nt=100, adv=FAKE, w=None, scale=1.0, low=0.2, high=0.28, dual=10.0,
             grad=FAKE, loss=FAKE, ws=FAKE, wsb=1 << 30):
        return L.pace_policy_loss(new, beh, tags, off, n, nt, adv, w, scale, low, high, dual, grad, loss, None, None, ws, wsb, None)

    for kw in (dict(new=None), dict(beh=None), dict(off=None), dict(off=FAKE + 4), dict(n=-1), dict(nt=-1), dict(nt=2 ** 40),
               dict(adv=None), dict(scale=float("nan")), dict(low=1.0), dict(low=-0.1), dict(high=-0.1), dict(high=float("nan")),
               dict(dual=1.0), dict(dual=float("nan")), dict(grad=None), dict(loss=None), dict(tags=FAKE + 2), dict(w=FAKE + 1)):
        assert call(**kw) == -1, kw
    for kw in (dict(ws=None), dict(ws=FAKE + 8), dict(wsb=128)):
        assert call(**kw) == -2, kw


def test_quantize_and_matmul_i8_host_argument_errors(L):
    def quant(x=FAKE, dt=0, n=4, k=100, st=100, q=FAKE, s=FAKE):
        return L.pace_quantize_rows(x, dt, n, k, st, q, s, None)

    for kw in (dict(x=None), dict(x=FAKE + 2), dict(dt=5), dict(n=-1), dict(k=0), dict(st=99), dict(q=None), dict(s=None), dict(s=FAKE + 2)):
        assert quant(**kw) == -1, kw

    def mul(a=FAKE, lda=64, sa=FAKE, b=FAKE, ldb=64, sb=FAKE, m=4, n=6, k=64, out=FAKE, dt=0, ldo=6, ws=FAKE, wsb=1 << 30):
        return L.pace_matmul_i8(a, lda, sa, b, ldb, sb, m, n, k, out, dt, ldo, ws, wsb, None)

    for kw in (dict(a=None), dict(b=None), dict(sa=None), dict(sb=None), dict(sa=FAKE + 1), dict(lda=63), dict(ldb=63), dict(m=-1),
               dict(n=-1), dict(k=0), dict(k=131072, lda=131072, ldb=131072), dict(out=None), dict(dt=3), dict(ldo=5),
               dict(out=FAKE + 2), dict(m=2 ** 30, n=2 ** 20, ldo=2 ** 20)):
        assert mul(**kw) == -1, kw
    for kw in (dict(ws=None), dict(ws=FAKE + 16), dict(wsb=8)):
        assert mul(**kw) == -2, kw


def test_orthogonalize_host_argument_errors(L):
    import ctypes
    coefs = (ctypes.c_double * 3)(1.5, -0.5, 0.0)
    nan = (ctypes.c_double * 3)(1.5, float("nan"), 0.0)

    def call(g=FAKE, dt=0, batch=2, rows=30, cols=40, st=40, bst=1200, steps=5, co=coefs, eps=1e-7, out=FAKE, ws=FAKE, wsb=1 << 30):
        return L.pace_orthogonalize(g, dt, batch, rows, cols, st, bst, steps, co, eps, out, ws, wsb, None)

    for kw in (dict(g=None), dict(g=FAKE + 2), dict(dt=3), dict(batch=-1), dict(batch=65536), dict(rows=0), dict(cols=0),
               dict(cols=2 ** 21 + 1, st=2 ** 22, bst=2 ** 40), dict(st=39), dict(bst=1199), dict(steps=-1), dict(steps=101), dict(co=None),
               dict(co=nan), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("inf")), dict(eps=float("nan")), dict(out=None), dict(out=FAKE + 1)):
        assert call(**kw) == -1, kw
    for kw in (dict(ws=None), dict(ws=FAKE + 32), dict(wsb=100)):
        assert call(**kw) == -2, kw


def test_gpu_tests_reach_every_tile():
    """The sizes of the GPU tests of tiles, by the library's own rule for a chip of 256 CUs."""
    from tests.operator_rules import CUS, rules
    from tests.test_gpu_matmul_i8 import TILES as I8
    from tests.test_gpu_orthogonalize import TILES as ORTHO
    R = rules()
    every = {64, 128, 192, 256}
    assert {R.full(m, n, 1, k // 128, CUS) for m, n, k in I8} == every
    gram, square, apply = set(), set(), set()
    for b, r, c in ORTHO:
        m, n = min(r, c), max(r, c)
        gram.add(R.lower(m, b, -(-n // 64), CUS))
        square.add(R.lower(m, b, -(-m // 64), CUS))
        apply.add(R.full(m, n, b, -(-m // 64), CUS))
    assert apply == every and gram >= {64, 128, 192} and square >= {64, 128, 192}, (gram, square, apply)


def test_logprob_parts_and_loss_spans():
    from tests.operator_rules import rules
    R = rules()
    for rows in (1, 2, 48, 300, 2048, 5000):
        for vocab in (1, 8191, 16384, 150000, 10 ** 6):
            for k in (0, 20, 64):
                p, w = R.parts(rows, vocab, k), R.waves(rows, vocab, k)
                assert w in (1, 8) and 1 <= p <= 64 and (p == 1 or vocab // p >= 4096)
                assert w == 8 or (k <= 32 and vocab // p <= 16384)
    for nt in (0, 1, 10 ** 6, 10 ** 8, 2 ** 40 - 1):
        s = R.span(nt)
        assert s >= 256 and s % 256 == 0 and nt // s <= 2 ** 31 - 2


def test_product_parts():
    """Splitting a product's steps: no part without a step, no more workgroups than the chip holds, and the GPU tests reach
    parts of one length and of two, in both kinds of workgroup."""
    from tests.operator_rules import CUS, rules
    from tests.test_gpu_matmul_i8 import PARTS as I8
    from tests.test_gpu_orthogonalize import PARTS as ORTHO
    R = rules()
    for steps in (1, 23, 24, 31, 47, 64, 125, 1000, 2 ** 15):
        for tiles in (1, 3, 10, 64, 136, 170, 171, 512, 10 ** 6):
            p = R.product(steps, tiles)
            run = -(-steps // p)
            assert p == 1 or (3 <= p <= 16 and p * tiles <= 512 and run >= 8 and (p - 1) * run < steps <= p * run)
            assert p == 1 or steps >= 24
    for jobs in ([(k // 128, -(-m // 64) * -(-n // 64)) for m, n, k in I8],
                 [(-(-max(r, c) // 64), (-(-min(r, c) // 64)) * (-(-min(r, c) // 64) + 1) // 2 * b) for b, r, c in ORTHO]):
        parts = [R.product(s, t) for s, t in jobs]
        assert min(parts) > 1
        assert {s % p == 0 for (s, _), p in zip(jobs, parts)} == {True, False}
        assert {t * p > CUS for (_, t), p in zip(jobs, parts)} == {True, False}


def test_gpu_tests_reach_every_small_step():
    from tests.operator_rules import CUS, rules
    from tests.test_gpu_orthogonalize import SMALL, WHOLE
    R = rules()
    got = set()
    for b, r, c in SMALL:
        mp, np = -(-min(r, c) // 64) * 64, -(-max(r, c) // 64) * 64
        assert not R.whole(mp, np)
        got.add((mp, R.cols(mp, max(r, c), b, CUS)))
    assert got == {(64, 64), (128, 64), (192, 64), (192, 128), (256, 64), (256, 128)}
    whole = {(-(-min(r, c) // 64) * 64, -(-max(r, c) // 64) * 64) for b, r, c in WHOLE}
    assert all(R.whole(*k) for k in whole) and {(64, 64), (64, 512), (128, 128), (128, 256)} <= whole
    # what a workgroup's threads and LDS hold
    assert all(mp * np <= 2 ** 15 and 4 * mp * np + 2 * mp * mp <= 160 * 1024
               for mp in range(64, 2049, 64) for np in range(mp, 4097, 64) if R.whole(mp, np))
    assert R.cols(128, 1000, 160, CUS) == 0 and R.cols(256, 300, 80, CUS) == 0 and R.cols(320, 320, 1, CUS) == 0
