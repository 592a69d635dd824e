"""GPU tests of workspaces kept for the largest problem: smaller ones run in them, with the same results, and a call
asks for no workspace that it does not use."""
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
    return pace


def space(size):
    return torch.full((size,), 255, dtype=torch.uint8, device=DEV)


def test_product(pace):
    say("i8 products in one workspace")
    ws = space(pace.pace_matmul_i8_workspace_bytes(300, 4096, 8192))
    b, sb = torch.randint(-128, 128, (4096, 8192), device=DEV, dtype=torch.int8), torch.rand(4096, device=DEV)
    for m in (1, 4, 7, 9, 16, 100, 128, 300):
        a, sa = torch.randint(-128, 128, (m, 8192), device=DEV, dtype=torch.int8), torch.rand(m, device=DEV)
        for n in (300, 4096):
            assert torch.equal(pace.pace_matmul_i8(a, sa, b[:n], sb[:n], workspace=ws), pace.pace_matmul_i8(a, sa, b[:n], sb[:n]))


def test_few_tokens_take_no_workspace(pace):
    say("i8 products of few tokens in 256 bytes")
    b, sb = torch.randint(-128, 128, (4096, 8192), device=DEV, dtype=torch.int8), torch.rand(4096, device=DEV)
    for m in (1, 3, 8):
        a, sa = torch.randint(-128, 128, (m, 8192), device=DEV, dtype=torch.int8), torch.rand(m, device=DEV)
        assert pace.pace_matmul_i8_workspace_bytes(m, 4096, 8192) == 256
        assert torch.equal(pace.pace_matmul_i8(a, sa, b, sb, workspace=space(256)), pace.pace_matmul_i8(a, sa, b, sb))
    with pytest.raises(pace.PaceError):              # sixteen are formed in parts
        pace.pace_matmul_i8(a.repeat(2, 1), sa.repeat(2), b, sb, workspace=space(256))


def test_policy_loss(pace):
    say("policy losses in one workspace")
    ws = space(pace.pace_policy_loss_workspace_bytes(3, 2200000))
    for nt in (1000, 2100000, 2105343, 2200000):
        lp, off, adv = torch.randn(nt, device=DEV), torch.tensor([0, nt // 3, nt // 2, nt], device=DEV), torch.randn(3, device=DEV)
        b = dict(pace.policy_loss_buffers(3, nt, DEV), workspace=ws)
        ref = pace.pace_policy_loss(lp, lp.flip(0), off, adv)
        assert all(torch.equal(x, y) for x, y in zip(pace.pace_policy_loss(lp, lp.flip(0), off, adv, buffers=b), ref))


def test_orthogonalize(pace):
    say("orthogonalised updates in one workspace")
    ws = space(pace.pace_orthogonalize_workspace_bytes(3, 1000, 4000))
    for batch, rows, cols in ((3, 1000, 4000), (1, 1000, 4000), (2, 256, 4000), (1, 64, 4000), (3, 900, 900), (3, 30, 40)):
        g = torch.randn(batch, rows, cols, device=DEV)
        assert torch.equal(pace.pace_orthogonalize(g, workspace=ws), pace.pace_orthogonalize(g))
