"""GPU test of the backward pass of pace_token_logprob where its row factors are large: masked tokens have no gradient,
whatever the factor of the entropy's.

Tolerance: the module test_gpu_logprob.py's, |dz error| <= |p part| ((T + 64) u + 8 u (|log p| + 2)) + 2 u |dz|, with
u = 2^-24 and T = vocab / 512 + 32."""
import math
import sys

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


@pytest.mark.parametrize("vocab", [40, 5000, 40001])
@pytest.mark.parametrize("mask", [-math.inf, torch.finfo(torch.float32).min])
@pytest.mark.parametrize("temperature,factor", [(1.0, 1.0), (1.0, 2e9), (1e-6, 1000.0), (1e-6, -1e12), (1e6, 1e20)])
def test_masked_tokens_have_no_gradient(pace, temperature, factor, mask, vocab):
    say("logprob backward, entropy's factor %g at temperature %g, vocab %d" % (factor, temperature, vocab))
    gen = torch.Generator(device=DEV).manual_seed(vocab)
    z = temperature * torch.randn(4, vocab, generator=gen, device=DEV)
    z[:, 3::4] = mask
    ids = torch.tensor([0, 1, 2, 4], dtype=torch.int32, device=DEV)
    g, gh = torch.randn(4, generator=gen, device=DEV), torch.full((4,), factor, device=DEV)
    _, ent, stats, _, _ = pace.pace_token_logprob(z, ids, temperature)
    dz = pace.pace_token_logprob_backward(z, ids, stats, g, ent, gh, temperature).double()
    assert not bool(dz[:, 3::4].any())
    lp = torch.log_softmax(z.double() / temperature, 1)
    p = lp.exp()
    far = p == 0
    plp = torch.where(far, 0.0, p * lp)
    h = -plp.sum(1, keepdim=True)
    one = torch.zeros_like(p).scatter_(1, ids.long()[:, None], 1.0)
    want = (g.double()[:, None] * (one - p) - gh.double()[:, None] * (plp + p * h)) / temperature
    part = (g.double().abs()[:, None] * p + gh.double().abs()[:, None] * p * (torch.where(far, 0.0, lp.abs()) + h)) / temperature
    tol = part * ((vocab / 512 + 96) * U + 8 * U * (torch.where(far, 0.0, lp.abs()) + 2)) + 2 * U * want.abs() + 1e-38
    assert float(((dz - want).abs() - tol).max()) <= 0
