"""GPU test of pace_token_logprob and its backward pass from the lowest temperature to the highest, every output.

Tolerances are those that test_gpu_logprob.py derives, which hold at any temperature: the difference to the largest
logit is taken before the division, so an error is relative to the log-probability, not to the logits over the
temperature. Two things go by the type's range: a log-probability below the least binary32 number is -inf, and a p
below 2^-126 counts as 0, which takes 2^-126 (|g| + |g_H| (|log p| + H)) / temperature from its gradient at most."""
import pytest

from tests.test_gpu_logprob import DEV, HALF_ULP, TINY, U, close, make, pace, reference, say, size  # noqa: F401  (pace is the fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [301, 2001, 40001])
@pytest.mark.parametrize("temperature", [1e-6, 1e-3, 0.05, 30.0, 1e3, 1e6])
def test_temperatures(pace, temperature, vocab, dtype):  # noqa: F811
    say("logprob temperature %g, %s, vocab %d" % (temperature, dtype, vocab))
    z, ids = make(7, vocab, dtype, 5)
    z[1] = torch.finfo(dtype).min
    ids[2] = int(z[2].argmax())                      # a log-probability near 0
    z[3, ::2] = torch.finfo(dtype).min
    z[4] = z[4] + 300.0
    z[5, vocab // 2] = z[5].max() + 3e-5             # close to the next ones
    ids[5] = vocab // 2
    gen = torch.Generator().manual_seed(0)
    g, ge = torch.randn(7, generator=gen), torch.randn(7, generator=gen)
    logp, ent, stats, top_ids, top_logp = pace.pace_token_logprob(z, ids, temperature, 4)
    dz = pace.pace_token_logprob_backward(z, ids, stats, g.to(DEV), ent, ge.to(DEV), temperature)
    ref = reference(z.cpu(), ids.cpu(), temperature, 4, g, ge)
    terms, lse = (vocab / 512 + 96) * U, ref["lse"]
    in_type = lambda x: torch.where(x.float() == -torch.inf, -torch.inf, x)
    for name, got, want, more in (("logp", logp, ref["logp"], lse), ("top_logp", top_logp, ref["top_logp"], lse[:, None])):
        close(name, got, in_type(want), terms + 8 * U * (size(want) + more))
    close("entropy", ent, ref["entropy"], terms * (2 + 2 * ref["entropy"]) + 8 * U * lse)
    assert torch.equal(top_ids.cpu(), ref["top_ids"])
    lp = ref["lp"].abs()
    none = 2.0 ** -126 * (g.abs()[:, None] + ge.abs()[:, None] * (lp + ref["entropy"][:, None])) / temperature
    tol = ref["part"] * (terms + 8 * U * (lp + 2)) + (ref["dz"].abs() + ref["part"] * U) * 2 * HALF_ULP[dtype] + TINY[dtype] + none
    close("dz", dz, ref["dz"], tol)
