"""GPU tests of pace_token_logprob where a workgroup of eight waves takes a row, or a part of one, in several rounds:
many long rows, which the other tests' shapes leave to the kernel of a wave a row. test_operators_plans_host.py holds
the shapes against the rule.

The reference is the definition in binary64, on the GPU; tolerances are those of test_gpu_logprob.py, u = 2^-24 and
T = vocab / 512 + 32: |logp error| <= (T + 64) u + 8 u (|logp| + log S), |entropy error| <= (T + 64) u (2 + 2 H) +
8 u log S, |dz error| <= |p part| ((T + 64) u + 8 u (|log p| + 2)) + 2 half units of the type of |dz| + |p part| u."""
import math
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 1e-38, torch.bfloat16: 1e-38, torch.float16: 2.0 ** -25}

# Rows that a workgroup takes whole, and in parts, by their number: (rows, vocabulary, alternatives).
WHOLE = [(4097, 33001, 0), (4097, 33001, 20), (2049, 20003, 64), (2049, 9001, 33)]
PARTS = [(1500, 70001, 0), (1025, 70001, 20), (700, 70001, 64), (40, 70001, 64), (3, 1200007, 20), (1, 2400001, 0)]


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


def best(z, k):
    """The k first ids in the order (logit descending, id ascending), by keys that are all different."""
    bits = (z.float() + 0.0).view(torch.int32).long()
    key = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits) * (1 << 31) + (z.shape[1] - 1 - torch.arange(z.shape[1], device=DEV))
    return z.shape[1] - 1 - (key.topk(k, 1).values & 0x7FFFFFFF)


def check(pace, z, ids, k, gh, seed):
    """Every row's outputs, 64 rows at a time."""
    n, vocab = z.shape
    gen = torch.Generator(device=DEV).manual_seed(seed)
    g = torch.randn(n, generator=gen, device=DEV)
    ge = torch.randn(n, generator=gen, device=DEV) if gh else None
    logp, ent, stats, top_ids, top_logp = pace.pace_token_logprob(z, ids, 1.0, k)
    dz = pace.pace_token_logprob_backward(z, ids, stats, g, ent if gh else None, ge)
    terms = (vocab / 512 + 96) * U
    for r in range(0, n, 64):
        s = slice(r, r + 64)
        live, t = ids[s] != -1, ids[s].long().clamp(min=0)[:, None]
        x = z[s].double()
        none = (x == -math.inf).all(1)
        x = torch.where((none | ~live)[:, None], 0.0, x)          # compared apart, below
        lse = torch.logsumexp(x - x.amax(1, keepdim=True), 1)
        lp = torch.log_softmax(x, 1)
        p = lp.exp()
        far = p == 0
        plp = torch.where(far, 0.0, p * lp)
        h = -plp.sum(1)
        rows = live & ~none
        w = lp.gather(1, t)[:, 0]
        masked = w == -math.inf
        assert bool((logp[s][rows & masked] == -math.inf).all())
        ok = rows & ~masked
        assert bool(((logp[s].double() - w).abs() <= terms + 8 * U * (w.abs() + lse))[ok].all())
        assert bool(((ent[s].double() - h).abs() <= terms * (2 + 2 * h) + 8 * U * lse)[rows].all())
        assert not bool(logp[s][~live].any()) and not bool(ent[s][~rows].any()) and bool((logp[s][live & none] == -math.inf).all())
        if k:
            b = best(z[s], k)
            v = z[s].gather(1, b)
            absent = (v == -math.inf) | ~live[:, None]
            assert torch.equal(top_ids[s], torch.where(absent, -1, b).to(torch.int32))
            tl = lp.gather(1, b)
            assert bool((top_logp[s][absent] == -math.inf).all())
            assert bool((((top_logp[s].double() - tl).abs() <= terms + 8 * U * (tl.abs() + lse[:, None])) | absent)[rows].all())
        one = torch.zeros_like(p).scatter_(1, t, 1.0)
        size = torch.where(far, 0.0, lp.abs())
        want = g[s].double()[:, None] * (one - p)
        part = (g[s].double()[:, None] * p).abs()
        if gh:
            want = want - ge[s].double()[:, None] * (plp + p * h[:, None])
            part = part + ge[s].double().abs()[:, None] * p * (size + h[:, None])
        want, part = (torch.where(rows[:, None], v, 0.0) for v in (want, part))
        tol = part * (terms + 8 * U * (size + 2)) + (want.abs() + part * U) * 2 * HALF_ULP[z.dtype] + TINY[z.dtype]
        assert bool(((dz[s].double() - want).abs() <= tol).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,vocab,k", WHOLE + PARTS)
def test_many_rounds(pace, dtype, n, vocab, k):
    say("logprob by workgroups %s n=%d vocab=%d k=%d" % (dtype, n, vocab, k))
    gen = torch.Generator(device=DEV).manual_seed(n + vocab)
    z = torch.empty(n, vocab, device=DEV).normal_(0.0, 2.5, generator=gen).to(dtype)
    ids = torch.randint(0, vocab, (n,), generator=gen, device=DEV, dtype=torch.int32)
    if n > 3:
        ids[::5] = -1
    check(pace, z, ids, k, gh=n % 2 == 1, seed=n)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n,vocab,k", [(4097, 33001, 20), (2049, 9001, 64), (1025, 70001, 20)])
def test_special_rows(pace, dtype, n, vocab, k):
    """Equal logits, which overflow the list of candidates, rising and falling ones, masks in places of every wave and
    round, one token left at either end, nothing left, a maximum in the last elements behind the vectors, off alignment."""
    say("logprob by workgroups, special rows %s n=%d vocab=%d k=%d" % (dtype, n, vocab, k))
    gen = torch.Generator(device=DEV).manual_seed(vocab)
    wide = torch.full((n, vocab + 3), float("nan"), dtype=dtype, device=DEV)
    z = wide[:, 1:1 + vocab]
    z.copy_(torch.empty(n, vocab, device=DEV).normal_(0.0, 2.5, generator=gen))
    ids = torch.randint(0, vocab, (n,), generator=gen, device=DEV, dtype=torch.int32)
    low = torch.finfo(dtype).min
    z[0] = float("nan"); ids[0] = -1
    z[1] = 1.5
    z[2] = torch.linspace(-8, 8, vocab, device=DEV).to(dtype)
    z[3] = torch.linspace(8, -8, vocab, device=DEV).to(dtype)
    z[4, 5:] = -math.inf; ids[4] = 2
    z[5, :vocab - 3] = -math.inf; ids[5] = vocab - 1
    z[6] = -math.inf
    z[7, vocab // 3:] = low; ids[7] = 1
    z[8] = low
    z[9, 1:] = -math.inf; ids[9] = 2                   # the given token itself is masked out
    z[10] = -math.inf; z[10, vocab - 1] = 3.0; ids[10] = vocab - 1
    z[11, vocab - 1] = 20.0
    z[12] = 0.0; z[12, ::2] = -0.0                     # ties
    z[13, ::3] = -math.inf; ids[13] = 1
    z[14] = -3.0; z[14, ::512] = 4.0                   # one thread holds every large one
    check(pace, z, ids, k, gh=True, seed=k)
