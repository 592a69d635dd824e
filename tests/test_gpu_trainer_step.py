"""The example of a trainer step: its parts against the plain formulas in 64 bits,
and that the policy learns."""
import importlib.util
import os
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def say(msg):
    sys.stdout.write("[gpu] %s\n" % msg)
    sys.stdout.flush()


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_36830_amd import _lib
    if not os.path.exists(_lib.library_path):
        from paper_2609_36830_amd import build
        build.build()
    spec = importlib.util.spec_from_file_location("trainer_step", os.path.join(ROOT, "examples", "trainer_step.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


LENGTHS = [1, 40, 7, 96, 33, 64, 2, 120, 81, 50, 35, 77]


def test_rollout_log_probs(example):
    """Behaviour log-probabilities are those of the served 8-bit heads, each token by the head that wrote it."""
    say("trainer step: rollout")
    t = example.Trainer(LENGTHS, hidden=192, vocab=1001, lag=2, seed=3)
    for _ in range(3):
        t.publish()
        pool = t.rollout()
        t.train(pool)
    t.publish()
    pool = t.rollout()
    wrote = pool["tags"].cpu()
    assert wrote.max() == 3 and set(wrote.tolist()) <= {-1, 1, 2, 3}
    x = pool["states"].double().cpu()
    for version, (q, scale) in t.served.items():
        rows = (wrote == version).nonzero()[:, 0]
        most = x[rows].abs().amax(1, keepdim=True)
        codes = (x[rows].float() * (127.0 * (1.0 / most.float()))).round().double()
        z = codes @ q.cpu().double().t() * (most / 127.0 * scale.cpu().double())
        lp = z.log_softmax(1)[torch.arange(len(rows)), pool["tokens"].cpu()[rows].long()]
        # logits are rounded to bfloat16: half an ulp each way of the token's and of the sum's
        near = 2 * 2.0 ** -8 * z.abs().amax(1) + 1e-4
        assert ((pool["lp_behavior"].cpu()[rows].double() - lp).abs() <= near).all()


def test_gradient_and_update(example):
    """The head's gradient against differentiating the loss in 64 bits; the update's singular values."""
    say("trainer step: gradient and update")
    t = example.Trainer(LENGTHS, hidden=192, vocab=1001, lag=2, seed=5, momentum=0.0)
    for _ in range(2):
        t.publish()
        t.train(t.rollout())
    t.publish()
    pool = t.rollout()
    head = t.head.to(torch.bfloat16).double().cpu().requires_grad_()
    r = t.train(pool)
    ids = t.step.kept_ids[: r["kept"]].cpu().long()
    off, reward = t.offsets.cpu(), pool["reward"].cpu().double()[ids]
    assert r["kept"] == 9 and r["tokens"] == int((off[ids + 1] - off[ids]).sum())
    advantage = (reward - reward.mean()) / (reward.std() + 1e-6)
    rows = torch.cat([torch.arange(off[i], off[i + 1]) for i in ids.tolist()])
    adv = torch.repeat_interleave(advantage, off[ids + 1] - off[ids])
    tags, tokens = pool["tags"].cpu()[rows], pool["tokens"].cpu()[rows].long()
    counts = tags >= 0
    x = pool["states"].cpu().double()[rows]
    lp = (x @ head.t()).log_softmax(1)[torch.arange(len(rows)), tokens]
    d = lp - pool["lp_behavior"].cpu().double()[rows]
    ratio = d.exp()
    up = torch.minimum(ratio, torch.tensor(1.28, dtype=torch.float64))
    down = torch.minimum(torch.maximum(ratio, torch.tensor(0.8, dtype=torch.float64)), torch.tensor(10.0, dtype=torch.float64))
    loss = -(adv * torch.where(adv > 0, up, down) * counts).sum() / counts.sum()
    loss.backward()
    # The logits and their gradient are bfloat16: 2^-9 of |z| (at most about 8) in each exponent, some 2% of a
    # probability at most, with random signs over the rows' sum; a token may change sides of a clip by as much.
    assert float((r["grad_head"].cpu().double() - head.grad).norm() / head.grad.norm()) < 0.05
    assert abs(r["loss"] - float(loss.detach())) < 0.02
    s = torch.linalg.svdvals(r["update"].double().cpu())
    assert s.max() < 1.3 and r["update"].shape == (1001, 192)


def test_policy_learns(example):
    """Eight steps raise the reward, the share of tokens of the vocabulary's lower half, from a half."""
    say("trainer step: learning")
    t = example.Trainer([64] * 64, lag=2, seed=0)
    rewards = []
    for _ in range(8):
        t.publish()
        rewards.append(t.train(t.rollout())["reward"])
    assert abs(rewards[0] - 0.5) < 0.1 and rewards[-1] > rewards[0] + 0.1
