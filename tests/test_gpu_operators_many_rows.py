"""GPU tests of the operators around the step on more rows, channels and trajectories than one launch's grid holds:
the outputs of one call are those of two calls on the halves, bit for bit, or the definition's."""
import sys

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
    yield pace
    torch.cuda.empty_cache()


def G(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def halves(n, call):
    h = n // 2
    return [torch.cat(p) for p in zip(call(slice(0, h)), call(slice(h, n)))]


def test_quantize_rows(pace):
    n = 2 ** 24 + 3
    say("quantize %d rows" % n)
    x = torch.randn(n, 3, generator=G(1), device=DEV).bfloat16()
    got = pace.pace_quantize_rows(x)
    assert all(torch.equal(a, b) for a, b in zip(got, halves(n, lambda s: pace.pace_quantize_rows(x[s]))))


@pytest.mark.parametrize("n,vocab,k", [(2 ** 26 + 9, 2, 0), (2 ** 23 + 3, 33, 33)])
def test_log_probabilities(pace, n, vocab, k):
    """A wave a row, and, for more than 32 alternatives, a workgroup."""
    say("log-probabilities of %d rows of %d" % (n, vocab))
    z = torch.randn(n, vocab, generator=G(2), device=DEV, dtype=torch.bfloat16)
    ids = torch.randint(-1, vocab, (n,), generator=G(3), device=DEV, dtype=torch.int32)
    got = pace.pace_token_logprob(z, ids, top_k=k)
    assert all(torch.equal(a, b) for a, b in zip(got, halves(n, lambda s: pace.pace_token_logprob(z[s], ids[s], top_k=k))))


@pytest.mark.parametrize("with_entropy", [False, True])
def test_backward(pace, with_entropy):
    n = 2 ** 24 + 5
    say("backward pass of %d rows" % n)
    z = torch.randn(n, 3, generator=G(4), device=DEV)
    ids = torch.randint(-1, 3, (n,), generator=G(5), device=DEV, dtype=torch.int32)
    g, gh = torch.randn(n, generator=G(6), device=DEV), torch.randn(n, generator=G(7), device=DEV)
    _, ent, stats, _, _ = pace.pace_token_logprob(z, ids)

    def call(s):
        return (pace.pace_token_logprob_backward(z[s], ids[s], stats[s], g[s], ent[s] if with_entropy else None,
                                                 gh[s] if with_entropy else None),)
    assert torch.equal(call(slice(None))[0], halves(n, call)[0])


def test_policy_loss(pace):
    """Trajectories without tokens but two of a thousand, which cross the spans of a wave."""
    n = 2 ** 26 + 5
    say("policy loss of %d trajectories" % n)
    off = torch.zeros(n + 1, dtype=torch.int64, device=DEV)
    off[n // 2:] = 1000
    off[n:] = 2000
    new, beh = torch.randn(2000, generator=G(8), device=DEV), torch.randn(2000, generator=G(9), device=DEV)
    b = pace.policy_loss_buffers(n, 2000, torch.device(DEV))
    for t in b.values():
        t.fill_(9)
    adv = torch.full((n,), -0.5, device=DEV)
    got = pace.pace_policy_loss(new, beh, off, adv, buffers=b)
    ref = pace.pace_policy_loss(new, beh, torch.tensor([0, 1000, 2000], device=DEV), adv[:2])
    assert torch.equal(got[0], ref[0])
    for a, c in zip(got[1:], ref[1:]):
        at = torch.tensor([n // 2 - 1, n - 1], device=DEV)
        assert torch.equal(a[at], c)
        a[at] = 0
        assert not bool(a.any())


@pytest.mark.parametrize("m,n", [(2, 2 ** 29 + 40), (9, 1620000000)])
def test_product_of_many_channels(pace, m, n):
    """Few tokens, and tiles, over rows of one byte: each output is one product, exact but for its scales."""
    say("i8 product of %d channels" % n)
    a = torch.randint(-128, 128, (m, 1), generator=G(10), device=DEV, dtype=torch.int8)
    b = torch.randint(-128, 128, (n, 1), generator=G(11), device=DEV, dtype=torch.int8)
    sa, sb = torch.rand(m, generator=G(12), device=DEV), torch.rand(n, generator=G(13), device=DEV)
    out = pace.pace_matmul_i8(a, sa, b, sb)
    step = 1 << 28
    for i in range(m):
        for j in range(0, n, step):
            s = slice(j, min(j + step, n))
            want = (a[i].float() * b[s, 0].float()) * (sa[i] * sb[s])
            assert torch.equal(out[i, s], want.bfloat16())
    del out, b, sb
    torch.cuda.empty_cache()
