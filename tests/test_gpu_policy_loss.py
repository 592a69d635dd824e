"""GPU tests of pace_policy_loss against a plain implementation in binary64.

Tolerances, u = 2^-24: the log ratio d is a binary32 number by definition and k
is rounded once (u); exp within 4u, one product (u): gradients and losses are
within 6u of their own size, the losses' sums (one sign within a trajectory,
binary64, rounded once) within 8u. The divergence term is a series of terms
within 10u for |d| < 0.7; beyond, (r - 1) - d with r within 4u and r at most
6.5 times the term: within 40u."""
import math
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


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


def D(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def reference(new, beh, off, adv, tags=None, weight=None, scale=1.0, low=0.2, high=0.28, dual=10.0):
    nt, n = len(new), len(off) - 1
    grad = np.zeros(nt)
    loss, kl, clipped = np.zeros(n), np.zeros(n), np.zeros(n, np.int64)
    with np.errstate(all="ignore"):
        lo, hi, far = (np.float32(v) for v in (math.log1p(-low), math.log1p(high), math.log(dual)))
        for i in range(n):
            s = slice(off[i], off[i + 1])
            k = scale * (1.0 if weight is None else float(weight[i])) * float(adv[i])
            d = new[s] - beh[s]                       # binary32
            live = np.ones(len(d), bool) if tags is None else tags[s] != -1
            r = np.exp(d.astype(np.float64))
            if k > 0:
                cut = d > hi
                l = -k * np.where(cut, 1 + high, r)
            elif k < 0:
                cut = (d < lo) | (d > far)
                l = -k * np.where(d < lo, 1 - low, np.where(d > far, dual, r))
            else:
                cut, l = np.zeros(len(d), bool), np.zeros(len(d))
            grad[s] = np.where(live & ~cut & (k != 0), -k * r, 0.0)
            loss[i] = l[live].sum()
            kl[i] = (np.expm1(d.astype(np.float64)) - d.astype(np.float64))[live].sum()
            clipped[i] = (cut & live).sum()
    return grad, loss, kl, clipped


def make(rng, lens, spread=0.2):
    off = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    nt = int(off[-1])
    beh = np.minimum(rng.normal(-1.2, 0.8, nt), 0).astype(np.float32)
    new = np.minimum(beh + rng.normal(0, spread, nt), 0).astype(np.float32)
    adv = rng.normal(0, 1, len(lens)).astype(np.float32)
    return off, new, beh, adv


def check(pace, off, new, beh, adv, tags=None, weight=None, **kw):
    names = {"clip_low": "low", "clip_high": "high", "dual_clip": "dual"}
    got = pace.pace_policy_loss(D(new), D(beh), D(off), D(adv), None if tags is None else D(tags),
                                None if weight is None else D(weight), **kw)
    ref = reference(new, beh, off, adv, tags, weight, **{names.get(k, k): v for k, v in kw.items()})
    g, loss, kl, clipped = (t.double().cpu().numpy() for t in got)
    for name, a, b, tol in (("grad", g, ref[0], 6 * U), ("loss", loss, ref[1], 8 * U), ("kl", kl, ref[2], 40 * U)):
        with np.errstate(over="ignore"):
            f = np.isfinite(b.astype(np.float32))     # e^90 is no binary32 number
        assert np.array_equal(np.isfinite(a), f), name
        assert np.all(np.abs(a[f] - b[f]) <= tol * np.abs(b[f]) + 1e-37), (name, np.max(np.abs(a[f] - b[f]) - tol * np.abs(b[f])))
    assert np.array_equal(clipped.astype(np.int64), ref[3])
    return got


@pytest.mark.parametrize("lens", [[1], [0], [0, 0, 3, 0], [255, 256, 257], [511, 512, 513, 1], [5000], [1, 100000, 1],
                                  [300] * 50, [1] * 700, [0] * 200 + [4] * 200 + [0] * 200, [70001, 0, 2, 30003]])
def test_lengths(pace, lens):
    say("policy loss lengths %s.. (%d)" % (lens[:4], len(lens)))
    rng = np.random.default_rng(len(lens))
    off, new, beh, adv = make(rng, lens)
    check(pace, off, new, beh, adv, scale=1.0 / max(1, off[-1]))
    tags = rng.integers(0, 9, off[-1]).astype(np.int32)
    tags[rng.random(off[-1]) < 0.4] = -1
    w = rng.random(len(lens)).astype(np.float32)
    check(pace, off, new, beh, adv, tags, w, scale=0.37)


def test_large_batch_spans_of_many_sizes(pace):
    """A batch whose spans are longer than the least, with trajectories longer and shorter than a span."""
    rng = np.random.default_rng(4)
    lens = np.concatenate([rng.integers(0, 12000, 900), [900000], rng.integers(0, 40, 3000)])
    say("policy loss %d tokens" % lens.sum())
    off, new, beh, adv = make(rng, lens)
    tags = np.where(rng.random(off[-1]) < 0.3, -1, 5).astype(np.int32)
    check(pace, off, new, beh, adv, tags, scale=1.0 / off[-1])


def test_bounds_and_special_values(pace):
    """Ratios at, just inside and just beyond every bound; infinities; advantage zero; NaN in masked places only."""
    say("policy loss bounds")
    at = [np.float32(v) for v in (math.log1p(-0.2), math.log1p(0.28), math.log(10.0))]
    d = np.array([x for v in at for x in (np.nextafter(v, np.float32(-9)), v, np.nextafter(v, np.float32(9)))] + [0.0, 3.0, -5.0, 90.0, -200.0],
                 np.float32)
    new, beh = np.tile(d, 3), np.zeros(3 * len(d), np.float32)
    off = np.array([0, len(d), 2 * len(d), 3 * len(d)], np.int64)
    check(pace, off, new, beh, np.array([1.5, -0.75, 0.0], np.float32))
    check(pace, off, new, beh, np.array([1.5, -0.75, 0.0], np.float32), clip_high=float("inf"), dual_clip=1e30)
    check(pace, off, new, beh, np.array([1.5, -0.75, 0.0], np.float32), clip_low=0.0, clip_high=0.0, dual_clip=1.0001)
    check(pace, off, new, beh, np.array([1.0, -1.0, -0.0], np.float32), scale=-2.0)
    new[3] = -np.inf                                  # a token that the new policy rules out
    new[len(d) + 3] = -np.inf
    check(pace, off, new, beh, np.array([1.5, -0.75, 1.0], np.float32))
    tags = np.zeros(len(new), np.int32)
    tags[::3] = -1
    new[::3], beh[::6] = np.nan, np.inf
    check(pace, off, new, beh, np.array([1.5, -0.75, 1.0], np.float32), tags)
    everything = np.full(len(new), -1, np.int32)     # masks that leave nothing
    got = check(pace, off, np.full_like(new, np.nan), beh, np.array([1.5, -0.75, 1.0], np.float32), everything)
    assert not bool(got[0].any()) and not bool(got[1].any())


def test_columns_wider_than_the_batch(pace):
    """Columns of full capacity, as pace_compact leaves them: behind offsets[n] nothing is read and gradients are 0."""
    say("policy loss behind the batch")
    rng = np.random.default_rng(8)
    off, new, beh, adv = make(rng, [700, 0, 1300])
    pad = np.full(5001, np.nan, np.float32)
    got = pace.pace_policy_loss(D(np.concatenate([new, pad])), D(np.concatenate([beh, pad])), D(off), D(adv))
    ref = pace.pace_policy_loss(D(new), D(beh), D(off), D(adv))
    assert torch.equal(got[0][:2000], ref[0]) and not bool(got[0][2000:].any())
    assert all(torch.equal(a, b) for a, b in zip(got[1:], ref[1:]))
    none = pace.pace_policy_loss(D(pad), D(pad), D(np.zeros(1, np.int64)), D(np.zeros(0, np.float32)))
    assert not bool(none[0].any())


@pytest.mark.parametrize("lead", [1, 2, 3])
def test_unaligned_starts(pace, lead):
    say("policy loss lead %d" % lead)
    rng = np.random.default_rng(9)
    off, new, beh, adv = make(rng, [1000, 37, 4000])
    tags = np.where(rng.random(off[-1]) < 0.3, -1, 5).astype(np.int32)
    ref = pace.pace_policy_loss(D(new), D(beh), D(off), D(adv), D(tags))

    def cut(x):
        return D(np.concatenate([np.zeros(lead, x.dtype), x]))[lead:]

    b = pace.policy_loss_buffers(3, off[-1], DEV)
    b["grad"] = torch.full((off[-1] + lead + 8,), 9.0, device=DEV)[lead:lead + off[-1]]
    got = pace.pace_policy_loss(cut(new), cut(beh), D(off), D(adv), cut(tags), buffers=b)
    assert all(torch.equal(a, c) for a, c in zip(got, ref))


def test_malformed_offsets_stay_in_bounds(pace):
    """Unspecified results, but nothing outside the outputs is written."""
    say("policy loss malformed offsets")
    rng = np.random.default_rng(10)
    new = rng.normal(0, 1, 4096).astype(np.float32)
    for off in ([5, 4000, 100, 9000], [-50, 10, 10, 1 << 40], [4096, 0, 4096, 0], [9, 8, 7, 6]):
        b = pace.policy_loss_buffers(3, 4096, DEV)
        guard = torch.full((4096 + 64,), 3.0, device=DEV)
        b["grad"] = guard[32:32 + 4096]
        pace.pace_policy_loss(D(new), D(new), D(np.array(off, np.int64)), D(np.ones(3, np.float32)), buffers=b)
        torch.cuda.synchronize()
        assert bool((guard[:32] == 3).all()) and bool((guard[-32:] == 3).all())


def test_gradient_against_differences(pace):
    """Central differences of the summed losses, away from the bounds: with step h = 2^-6 the third derivative |k| r
    (r < 1.3) gives h^2 / 4 |k|, the sums' rounding 8u sum|loss| / h, and d + h is exact to 2u."""
    say("policy loss gradient against differences")
    rng = np.random.default_rng(12)
    lens = [40, 33]
    off, new, beh, adv = make(rng, lens, 0.02)
    adv = np.array([0.8, -1.1], np.float32)
    h = np.float32(2.0 ** -6)
    g = pace.pace_policy_loss(D(new), D(beh), D(off), D(adv))[0].cpu().numpy()
    for t in (0, 17, 40, 72):
        i = 0 if t < 40 else 1
        up, down = new.copy(), new.copy()
        up[t] += h
        down[t] -= h
        lu, ld = (pace.pace_policy_loss(D(x), D(beh), D(off), D(adv))[1][i].item() for x in (up, down))
        num = (lu - ld) / (float(up[t]) - float(down[t]))
        tol = abs(adv[i]) * (h * h / 4 + 8 * U * 1.3 * lens[i] / h + 4 * U / h)
        assert abs(num - g[t]) <= tol


def test_follows_the_step_and_repeats(pace):
    """On a batch packed by pace_filter_step, repeated, on another stream and from a graph: the same bits."""
    import poolgen
    say("policy loss on the multiturn pool's batch")
    pool = poolgen.make_pool("multiturn")
    tags, off, comp = D(pool.tags), D(pool.offsets), D(pool.completion)
    step = pace.FilterStep(pool.n, pool.n_tokens, [torch.int32, torch.float32], DEV)
    gen = torch.Generator(device=DEV).manual_seed(3)
    beh = -torch.rand(pool.n_tokens, generator=gen, device=DEV)
    step.run(tags, off, comp, pool.V, pool.occupancy, pool.capacity, [tags, beh], D(pool.prefix_score), D(pool.window))
    n = pool.n - step.budget
    new = step.cols_out[1] + 0.1 * torch.randn(pool.n_tokens, generator=gen, device=DEV)
    adv = torch.randn(n, generator=gen, device=DEV)
    args = (new, step.cols_out[1], step.offsets_out[:n + 1], adv, step.cols_out[0])
    b = pace.policy_loss_buffers(n, pool.n_tokens, DEV)
    ref = [t.clone() for t in pace.pace_policy_loss(*args, scale=1e-6, buffers=b)]
    kept = int(step.n_kept_tokens.item())
    want = reference(new[:kept].cpu().numpy(), step.cols_out[1][:kept].cpu().numpy(), step.offsets_out[:n + 1].cpu().numpy(),
                     adv.cpu().numpy(), step.cols_out[0][:kept].cpu().numpy(), scale=1e-6)
    assert np.all(np.abs(ref[1].double().cpu().numpy() - want[1]) <= 8 * U * np.abs(want[1]))
    assert np.array_equal(ref[3].cpu().numpy(), want[3])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = pace.pace_policy_loss(*args, scale=1e-6, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(got, ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pace.pace_policy_loss(*args, scale=1e-6, buffers=b)
    for _ in range(3):
        for t in b.values():
            t.fill_(5)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(b[k], r) for k, r in zip(("grad", "loss", "kl", "clipped"), ref))


def test_refusals(pace):
    say("policy loss refusals")
    off, new, beh, adv = make(np.random.default_rng(1), [10, 20])
    a = dict(lp_new=D(new), lp_behavior=D(beh), offsets=D(off), advantage=D(adv))
    for kw in (dict(lp_new=a["lp_new"].double()), dict(lp_behavior=a["lp_behavior"][:5]), dict(advantage=a["advantage"][:1]),
               dict(tags=torch.zeros(30, dtype=torch.int64, device=DEV)), dict(weight=torch.ones(3, device=DEV)),
               dict(buffers=pace.policy_loss_buffers(1, 30, DEV)), dict(lp_new=a["lp_new"].cpu())):
        with pytest.raises(ValueError):
            pace.pace_policy_loss(**{**a, **kw})
    for kw in (dict(scale=float("inf")), dict(clip_low=1.0), dict(clip_low=-0.1), dict(clip_high=-1.0), dict(dual_clip=1.0)):
        with pytest.raises(pace.PaceError):
            pace.pace_policy_loss(**a, **kw)


def test_workspace_of_another_place_or_type(pace):
    """A workspace in host memory, or counted in another unit than bytes, is refused before anything runs."""
    f = lambda n: torch.zeros(n, device=DEV)
    for bad in (torch.empty(1 << 20, dtype=torch.uint8), torch.empty(1 << 18, dtype=torch.float32, device=DEV)):
        b = pace.policy_loss_buffers(1, 9, torch.device(DEV))
        with pytest.raises(ValueError):
            pace.pace_policy_loss(f(9), f(9), torch.tensor([0, 9], device=DEV), f(1), buffers=dict(b, workspace=bad))
