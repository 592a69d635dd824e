"""The example of a trainer step with a layer norm before the head: the operators together, against the plain formulas in
64 bits."""
import importlib.util
import os
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LENGTHS = [1, 40, 7, 96, 33, 64, 2, 120, 81, 50, 35, 77]


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


@pytest.mark.parametrize("bits", [32, 8])
def test_gradients_and_update(example, bits):
    """The gradients of head, weight and bias against differentiating the loss in 64 bits; the update of weight and bias
    from their gradients, clipped."""
    say("trainer step with a norm: gradients and update, %d bits" % bits)
    t = example.Trainer(LENGTHS, hidden=192, vocab=1001, lag=2, seed=5, momentum=0.0, norm=True, bits=bits, max_norm=0.01)
    for _ in range(2):
        t.publish()
        t.train(t.rollout())
    t.publish()
    pool = t.rollout()
    head = t.head.to(torch.bfloat16).double().cpu().requires_grad_()
    weight, bias = (p.double().cpu().requires_grad_() for p in t.norm)
    if bits == 8:
        import paper_2609_36830_amd as pace
        m, v = ([x.double().cpu() for x in xs] for xs in pace.pace_adamw_unpack(t.norm_state))
    else:
        m, v = ([x.double().cpu() for x in t.norm_state[k]] for k in ("exp_avg", "exp_avg_sq"))
    r = t.train(pool)
    ids = t.step.kept_ids[: r["kept"]].cpu().long()
    off, reward = t.offsets.cpu(), pool["reward"].cpu().double()[ids]
    advantage = (reward - reward.mean()) / (reward.std() + 1e-6)
    rows = torch.cat([torch.arange(off[i], off[i + 1]) for i in ids.tolist()])
    adv = torch.repeat_interleave(advantage, off[ids + 1] - off[ids])
    tags, tokens = pool["tags"].cpu()[rows], pool["tokens"].cpu()[rows].long()
    counts = tags >= 0
    x = pool["states"].cpu().double()[rows]
    h = torch.nn.functional.layer_norm(x, (192,), weight, bias, 1e-5)
    lp = (h @ head.t()).log_softmax(1)[torch.arange(len(rows)), tokens]
    ratio = (lp - pool["lp_behavior"].cpu().double()[rows]).exp()
    up = torch.minimum(ratio, torch.tensor(1.28, dtype=torch.float64))
    down = torch.minimum(torch.maximum(ratio, torch.tensor(0.8, dtype=torch.float64)), torch.tensor(10.0, dtype=torch.float64))
    loss = -(adv * torch.where(adv > 0, up, down) * counts).sum() / counts.sum()
    grads = torch.autograd.grad(loss, (head, weight, bias))
    # States after the norm, logits and their gradient are bfloat16, as in the test without a norm: random signs, some 2% of a
    # probability at most, and a token may change sides of a clip; the gradient to the states is rounded once more.
    for got, want in zip([r["grad_head"]] + r["grad_norm"], grads):
        assert float((got.cpu().double() - want).norm() / want.norm()) < 0.06
    # the update, from the gradients that the step had
    g = [x.cpu().double() for x in r["grad_norm"]]
    size = sum(float((x * x).sum()) for x in g) ** 0.5
    assert abs(r["grad_size"] - size) <= 1e-6 * size and size > 0.01           # clipped
    for k, p in enumerate((weight, bias)):
        d = g[k] * (0.01 / size)
        mk, vk = 0.9 * m[k] + (1 - 0.9) * d, 0.999 * v[k] + (1 - 0.999) * d * d
        want = p.detach() - 0.01 / (1 - 0.9 ** 3) * mk / ((vk / (1 - 0.999 ** 3)).sqrt() + 1e-8)
        # a step is at most some 0.01 / (1 - 0.9^3) times 1 / sqrt(0.001 / (1 - 0.999^3)), 0.06: 30 roundings of it, two of the parameter
        assert ((t.norm[k].cpu().double() - want).abs() <= 2.0 ** -24 * (2 * want.abs() + 30 * 0.06)).all()


def test_rollouts_go_through_the_norm(example):
    """Behaviour log-probabilities are those of the served version's norm and head."""
    say("trainer step with a norm: rollout")
    t = example.Trainer(LENGTHS, hidden=192, vocab=1001, lag=2, seed=3, norm=True, bits=8, norm_lr=0.1)
    for _ in range(3):
        t.publish()
        t.train(t.rollout())
    t.publish()
    pool = t.rollout()
    wrote = pool["tags"].cpu()
    for version, (q, scale) in t.served.items():
        rows = (wrote == version).nonzero()[:, 0]
        weight, bias = (p.double().cpu() for p in t.served_norm[version])
        h = torch.nn.functional.layer_norm(pool["states"].cpu().double()[rows], (192,), weight, bias, 1e-5)
        z = h @ (q.cpu().double() * scale.cpu().double()[:, None]).t()
        lp = z.log_softmax(1)[torch.arange(len(rows)), pool["tokens"].cpu()[rows].long()]
        # the states' bfloat16 (2^-8 of each) and 8 bits (half a step of most / 127, most at most 16): both with the signs of the
        # head's 192 entries, some 1 / 192^.5 each; then the logits' bfloat16, for the token and for the sum
        states = (2.0 ** -8 * h.abs() + h.abs().amax(1, keepdim=True) / 254) @ (q.cpu().double() * scale.cpu().double()[:, None]).abs().t()
        near = 2 * states.amax(1) + 2 * 2.0 ** -8 * z.abs().amax(1) + 1e-4
        assert ((pool["lp_behavior"].cpu()[rows].double() - lp).abs() <= near).all()
