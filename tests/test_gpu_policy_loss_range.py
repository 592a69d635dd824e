"""GPU test of pace_policy_loss at the ends of its exponential's range, without upper bounds.

Tolerances, u = 2^-24: r within 4u, k and one product u each: gradients and losses within 6u of their size. A divergence
of such a token is r less at most 90, beside which r is above 2^115: within 6u too; below, where r is nothing, 1 + d is
exact to 2u of it."""
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


@pytest.mark.parametrize("lo,hi", [(80.0, 88.722830), (-86.9, -80.0), (-110.0, -87.4)])
def test_exponential_at_the_ends(pace, lo, hi):
    say("policy loss for log ratios from %g to %g" % (lo, hi))
    d = np.unique(np.concatenate([np.linspace(lo, hi, 5001), [lo, hi]]).astype(np.float32))
    d = d[(d >= np.float32(lo)) & (d <= np.float32(hi))]
    adv = np.where(np.arange(len(d)) % 2, 0.75, -0.5).astype(np.float32)
    got = pace.pace_policy_loss(D(d), D(np.zeros_like(d)), D(np.arange(len(d) + 1)), D(adv), clip_low=0.0 if lo > 0 else 0.999, clip_high=math.inf,
                                dual_clip=math.inf)
    grad, loss, kl = (t.double().cpu().numpy() for t in got[:3])
    x = d.astype(np.float64)
    r = np.where(x < -87.35, 0.0, np.exp(x))
    tiny = np.where(x < -87.35, 2.0 ** -126, 0.0)    # as much or nothing
    cut = (adv < 0) & (lo < 0)                       # below the lower bound
    want = -adv * r
    assert np.all(np.abs(grad - np.where(cut, 0.0, want)) <= 6 * U * np.abs(want) + tiny)
    assert np.all(np.abs(loss - np.where(cut, 0.5 * (1.0 - 0.999), want)) <= 6 * U * np.abs(np.where(cut, 0.0005, want)) + tiny)
    z = np.expm1(x) - x if lo > 0 else -1.0 - x
    assert np.all(np.abs(kl - z) <= 6 * U * np.abs(z))
    assert np.array_equal(got[3].cpu().numpy(), cut.astype(np.int32))
