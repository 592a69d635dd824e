"""A trainer step around the filter: rollouts, rescoring, filter, loss, update.

A policy of a fixed body (random hidden states) and a learned head, float32
weights [vocab, hidden], answers prompts of random tokens:

1. rollout: log-probabilities of the sampled tokens from the head in 8 bits,
   by the weights of the version that wrote them;
2. rescoring: the Prefix Forgetting Score of the finished trajectories under
   the current head, in 8 bits;
3. the filter step rejects the stalest trajectories and packs the others;
4. training: logits in bfloat16, log-probabilities, the clipped loss, its
   gradient to the head, a momentum, and the orthogonalised update.

    python examples/trainer_step.py --steps 8
    python examples/trainer_step.py --steps 8 --norm --bits 8

With --norm a learned layer norm stands before the head, in rollouts, rescoring
and training; its weight and bias, which are no matrices, are updated by AdamW with
their gradients clipped, its moments in 32 bits or in 8.

The reward is the share of a trajectory's tokens below the vocabulary's middle,
so the policy learns to answer with those; each step prints one line.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2609_36830_amd as pace  # noqa: E402


class Trainer:
    """The policy and the buffers of pools of one shape: trajectories of the given lengths."""

    def __init__(self, lengths, hidden=256, vocab=4096, capacity=None, lag=2, lr=0.5, momentum=0.9, seed=0, device="cuda:0",
                 norm=False, bits=32, norm_lr=0.01, max_norm=1.0):
        self.dev = torch.device(device)
        self.gen = torch.Generator(self.dev).manual_seed(seed)
        self.lengths = torch.as_tensor(lengths, dtype=torch.int64).to(self.dev)
        self.n, self.n_tokens = len(lengths), sum(lengths)
        self.hidden, self.vocab, self.lag, self.lr, self.momentum = hidden, vocab, lag, lr, momentum
        self.capacity = self.n * 3 // 4 if capacity is None else capacity
        self.head = torch.randn(vocab, hidden, generator=self.gen, device=self.dev) * hidden ** -0.5
        self.velocity = torch.zeros_like(self.head)
        self.version, self.served, self.served_norm = 0, {}, {}
        self.norm, self.norm_lr, self.max_norm = None, norm_lr, max_norm
        if norm:
            self.norm = [torch.ones(hidden, device=self.dev), torch.zeros(hidden, device=self.dev)]      # weight, bias
            self.norm_state = pace.adamw_state(self.norm, bits)
        self.offsets = torch.cat([self.lengths.new_zeros(1), self.lengths.cumsum(0)])
        self.owner = torch.repeat_interleave(torch.arange(self.n, device=self.dev), self.lengths)
        self.at = torch.arange(self.n_tokens, device=self.dev) - self.offsets[self.owner]
        # what the calls of every step write, and their workspaces
        self.product = pace.matmul_i8_buffers(self.n_tokens, vocab, hidden, torch.bfloat16, self.dev)
        self.scored = pace.token_logprob_buffers(self.n_tokens, vocab, 0, self.dev)
        self.step = pace.FilterStep(self.n, self.n_tokens, [torch.int32, torch.int32, torch.float32, torch.int32], self.dev)
        self.update = pace.orthogonalize_buffers(1, vocab, hidden, self.dev)
        self.update["out"] = self.update["out"][0]
        self.clip = pace.grad_norm_buffers(2, 2 * hidden, self.dev)

    def publish(self):
        """The head as rollouts and rescoring serve it: 8 bits and a scale for each token's row, with the norm before it. Old
        versions go."""
        self.served[self.version] = pace.pace_quantize_rows(self.head)
        self.served_norm[self.version] = None if self.norm is None else [w.clone() for w in self.norm]
        self.served_norm.pop(self.version - self.lag - 1, None)
        self.served.pop(self.version - self.lag - 1, None)

    def logits(self, states, version):
        """Logits after the hidden states, by a served head; a whole pool's go to the kept buffers."""
        if self.norm is not None:
            states, _ = pace.pace_layer_norm(states, *self.served_norm[version])
        if states.shape[0] < self.n_tokens:
            return pace.pace_matmul_i8(*pace.pace_quantize_rows(states), *self.served[version])
        p = self.product
        q, scale = pace.pace_quantize_rows(states, q_out=p["q"], scale_out=p["scale"])
        return pace.pace_matmul_i8(q, scale, *self.served[version], out=p["out"], workspace=p["workspace"])

    def rollout(self):
        """A pool of finished trajectories, each begun up to `lag` versions ago and written by the next version from
        its middle on. Every seventh token comes from a tool, which no policy is scored for."""
        begun = self.version - torch.randint(0, min(self.lag, self.version) + 1, (self.n,), generator=self.gen, device=self.dev)
        wrote = (begun[self.owner] + (2 * self.at >= self.lengths[self.owner])).clamp_(max=self.version)
        states = torch.randn(self.n_tokens, self.hidden, generator=self.gen, device=self.dev).add_(1.0).to(torch.bfloat16)
        tokens = torch.empty(self.n_tokens, dtype=torch.int32, device=self.dev)
        lp = torch.empty(self.n_tokens, device=self.dev)
        for version in self.served:
            rows = (wrote == version).nonzero()[:, 0]
            z = self.logits(states[rows], version)
            noise = torch.rand(z.shape, generator=self.gen, device=self.dev).clamp_(min=1e-20)
            tokens[rows] = (z.float() - (-noise.log()).log()).argmax(1).to(torch.int32)
            lp[rows] = pace.pace_token_logprob(z, tokens[rows])[0]
        low = (tokens < self.vocab // 2).float()
        return dict(states=states, tokens=tokens, lp_behavior=lp,
                    tags=torch.where(self.at % 7 == 6, -1, wrote).to(torch.int32),
                    completion=wrote[(self.offsets[1:] - 1).clamp(min=0)].to(torch.int32),
                    reward=torch.zeros(self.n, device=self.dev).index_add_(0, self.owner, low) / self.lengths.clamp(min=1))

    def train(self, pool):
        """One step of the trainer over a finished pool."""
        # rescoring by the head of now
        lp_now, *_ = pace.pace_token_logprob(self.logits(pool["states"], self.version), pool["tokens"], buffers=self.scored)
        forgotten = pace.pace_prefix_score(lp_now, pool["lp_behavior"], self.offsets, pool["tags"])
        # the filter: the stalest are rejected, the others packed, with each token's place in the pool
        place = torch.arange(self.n_tokens, dtype=torch.int32, device=self.dev)
        window = forgotten[~forgotten.isnan()].sort().values
        step = self.step.run(pool["tags"], self.offsets, pool["completion"], self.version, self.n, self.capacity,
                             [pool["tags"], pool["tokens"], pool["lp_behavior"], place], prefix=forgotten, window=window)
        kept, n_tokens = self.n - step.budget, int(step.n_kept_tokens.item())
        tags, tokens, lp_behavior, place = (c[:n_tokens] for c in step.cols_out)
        offsets, reward = step.offsets_out[: kept + 1], pool["reward"][step.kept_ids[:kept].long()]
        advantage = (reward - reward.mean()) / (reward.std() + 1e-6)
        # the batch: a mean over its response tokens
        states = pool["states"][place.long()]
        scored = torch.where(tags >= 0, tokens, -1)
        response = max(int((tags >= 0).sum()), 1)
        head, hidden = self.head.to(torch.bfloat16), states
        if self.norm is not None:
            hidden, norm_stats = pace.pace_layer_norm(states, *self.norm)
        logits = hidden @ head.t()
        lp, entropy, stats, *_ = pace.pace_token_logprob(logits, scored)
        grad_lp, loss, kl, clipped = pace.pace_policy_loss(lp, lp_behavior, offsets, advantage, tags, scale=1.0 / response)
        grad_logits = pace.pace_token_logprob_backward(logits, scored, stats, grad_lp, grad_logits_out=logits)
        grad_head = (grad_logits.t() @ hidden).float()
        more = {}
        if self.norm is not None:
            _, *grads = pace.pace_layer_norm_backward(states, norm_stats, grad_logits @ head, self.norm[0])
            clipped_norm, factor = pace.pace_grad_norm(grads, self.max_norm, buffers=self.clip)
            # The default betas do for the few steps here; longer runs with moments in 8 bits want betas=(0.9, 0.95).
            pace.pace_adamw(self.norm, grads, self.norm_state, lr=self.norm_lr, step=self.version + 1, grad_scale=factor)
            more = dict(grad_norm=grads, grad_size=float(clipped_norm))
        self.velocity.mul_(self.momentum).add_(grad_head)
        update = pace.pace_orthogonalize(self.velocity, **self.update)
        self.head.add_(update, alpha=-self.lr)
        self.version += 1
        return dict(kept=kept, tokens=n_tokens, reward=float(pool["reward"].mean()), loss=float(loss.sum()),
                    kl=float(kl.sum()) / response, entropy=float(entropy.sum()) / response, clipped=int(clipped.sum()),
                    grad_head=grad_head, update=update, **more)


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--trajectories", type=int, default=64)
    ap.add_argument("--max-tokens", type=int, default=200)
    ap.add_argument("--lag", type=int, default=2, help="versions that a trajectory may be behind")
    ap.add_argument("--seed", type=int, default=0)
    ap.add_argument("--norm", action="store_true", help="a learned layer norm before the head")
    ap.add_argument("--bits", type=int, default=32, choices=(32, 8), help="of the moments of its weight and bias")
    args = ap.parse_args()
    lengths = torch.randint(1, args.max_tokens + 1, (args.trajectories,), generator=torch.Generator().manual_seed(args.seed))
    trainer = Trainer(lengths.tolist(), lag=args.lag, seed=args.seed, norm=args.norm, bits=args.bits)
    for k in range(args.steps):
        trainer.publish()
        r = trainer.train(trainer.rollout())
        print("step %d  kept %d of %d (%d tokens)  reward %.3f  loss %+.4f  kl %.5f  entropy %.3f  clipped %d" % (
            k, r["kept"], trainer.n, r["tokens"], r["reward"], r["loss"], r["kl"], r["entropy"], r["clipped"]), flush=True)


if __name__ == "__main__":
    main()
