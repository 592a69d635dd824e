"""GPU tests of the sums of pace_policy_loss by trajectory.

A trajectory of one token gives that token's own loss and divergence, binary32 numbers, so a longer trajectory's are
their binary64 sum rounded once. In binary64 the sum's order shows below 2^-40 of it: the bits are equal."""
import sys

import numpy as np
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


def D(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


@pytest.mark.parametrize("length", [2, 3, 4, 7, 64, 1000])
def test_sums_are_binary64(pace, length):
    say("policy loss sums of %d tokens" % length)
    rng = np.random.default_rng(length)
    n = max(40000 // length, 40)
    nt = n * length
    new = rng.normal(0, 0.7, nt).astype(np.float32)
    new[rng.random(nt) < 0.3] -= 12                  # terms of very different sizes
    beh = np.zeros(nt, np.float32)
    adv = rng.normal(0, 1, n).astype(np.float32)
    each = pace.pace_policy_loss(D(new), D(beh), D(np.arange(nt + 1)), D(np.repeat(adv, length)), dual_clip=1e4, clip_low=0.999999)
    whole = pace.pace_policy_loss(D(new), D(beh), D(np.arange(n + 1) * length), D(adv), dual_clip=1e4, clip_low=0.999999)
    for e, w in zip(each[1:3], whole[1:3]):
        want = e.double().view(n, length).sum(1)
        assert torch.equal(w, want.float())
    assert torch.equal(each[0], whole[0])
