"""Post-training a small model's output layer on what its answers earned.

A worked example of the training entry points as a program calls them
together, on synthetic contexts: the model is a bfloat16 output layer over
fixed hidden states, an answer is a request of a few tokens, and a token earns
a point when it is one of a quarter of the vocabulary.

- ``policy``: tokens are drawn with their features (:func:`sample_features`),
  the clipped policy loss writes its gradient over the logits, and AdamW
  steps the float32 weights and refreshes their bfloat16 copy.
- ``preference``: two answers are drawn for each context, the one that earned
  more is the chosen one, and the reference is the layer it started from.

Afterwards the answers are scored and routed as in serving.

    python -m paper_2608_28726_amd.post_train [policy|preference] [steps]
"""

from __future__ import annotations

import sys

import torch

import paper_2608_28726_amd as pr

TEMPERATURE = 1.0


class OutputLayer:
    """Float32 weights [vocab, width], the bfloat16 copy that computes with them, and their optimizer."""

    def __init__(self, vocab: int, width: int, state_bits: int, seed: int, device):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.weight = torch.empty(vocab, width, device=device).normal_(std=width ** -0.5, generator=g)
        self.copy = self.weight.bfloat16()
        self.opt = pr.AdamW([self.weight], copies=[self.copy], state_bits=state_bits, seed=seed)

    def logits(self, hidden):
        return hidden @ self.copy.t()

    def step(self, hidden, grad_logits, lr: float):
        """The product rule of the layer, then the optimizer's step."""
        self.opt.step(lr=lr, weight_decay=0.0, grads=[grad_logits.t() @ hidden])


def _policy_step(layer, hidden, earns, weight, length, lr, seed, step):
    logits = layer.logits(hidden)
    ids, feats, _ = pr.sample_features(logits, TEMPERATURE, seed, offset=step)
    reward = earns[ids.long()]
    per_request = reward.view(-1, length).mean(1)
    advantage = (per_request - per_request.mean()).repeat_interleave(length) + reward - reward.mean()
    out = pr.policy_loss(logits, ids, TEMPERATURE, weight, advantage, feats["logprob"], grad=logits)
    layer.step(hidden, out["grad"], lr)
    return out["loss"], reward.mean()


def _preference_step(layer, hidden, earns, weight, length, lr, seed, step, ref, offsets):
    n = hidden.shape[0] // 2  # rows of the pairs' first answers; the second ones have the same contexts
    logits = layer.logits(hidden)
    ids, _, _ = pr.sample_features(logits, TEMPERATURE, seed, offset=step, features=False)
    reward = earns[ids.long()]
    both = ids.view(2, -1, length), reward.view(2, -1, length)
    first = (both[1][0].sum(1) >= both[1][1].sum(1))[:, None]
    chosen, rejected = torch.where(first, both[0][0], both[0][1]), torch.where(first, both[0][1], both[0][0])
    ids = torch.stack([chosen, rejected], 1).reshape(-1).contiguous()
    rows = torch.stack([hidden[:n].view(-1, length, hidden.shape[1])] * 2, 1).reshape(2 * n, -1)
    logits = layer.logits(rows)
    before = pr.token_features(rows @ ref.t(), ids, TEMPERATURE)["logprob"]
    out = pr.preference_loss(logits, ids, TEMPERATURE, weight, offsets, before, grad=logits)
    layer.step(rows, out["grad"], lr)
    return out["loss"], reward.mean()


def post_train(method: str = "policy", steps: int = 60, vocab: int = 4096, width: int = 64, requests: int = 64,
               length: int = 8, lr: float = 0.02, state_bits: int = 8, seed: int = 0, device="cuda") -> dict:
    """Runs the example; returns the losses and mean rewards of the steps and the share of answers that would ship."""
    if method not in ("policy", "preference"):
        raise ValueError("method must be 'policy' or 'preference'")
    g = torch.Generator(device=device)
    g.manual_seed(seed + 1)
    n = requests * length
    hidden = torch.empty(n, width, device=device).normal_(generator=g)
    hidden[:, 0] = 2.0  # what every context has in common
    hidden = hidden.bfloat16()
    earns = (torch.rand(vocab, generator=g, device=device) < 0.25).float()
    layer = OutputLayer(vocab, width, state_bits, seed, device)
    offsets = torch.arange(0, n + 1, length, dtype=torch.int32, device=device)
    losses, rewards = [], []
    if method == "policy":
        weight = torch.full((n,), 1.0 / n, device=device)
        for step in range(steps):
            loss, reward = _policy_step(layer, hidden, earns, weight, length, lr, seed, step)
            losses.append(loss)
            rewards.append(reward)
    else:
        ref = layer.copy.clone()
        twice = torch.cat([hidden, hidden])
        weight = torch.ones(2 * n, device=device)
        pairs = torch.arange(0, 2 * n + 1, length, dtype=torch.int32, device=device)
        for step in range(steps):
            loss, reward = _preference_step(layer, twice, earns, weight, length, lr, seed, step, ref, pairs)
            losses.append(loss)
            rewards.append(reward)
    ids, feats, _ = pr.sample_features(layer.logits(hidden), TEMPERATURE, seed, offset=steps)
    score = pr.request_aggregate(feats, offsets)["score"]
    _, n_ship = pr.route(score, float(score.median()))
    return {"loss": torch.cat(losses).tolist(), "reward": torch.stack(rewards).tolist(),
            "reward_after": float(earns[ids.long()].mean()), "shipped": int(n_ship) / requests}


def main(argv) -> int:
    method = argv[0] if argv else "policy"
    steps = int(argv[1]) if len(argv) > 1 else 60
    out = post_train(method, steps)
    for k in range(0, steps, max(1, steps // 10)):
        print(f"step {k:4d}  loss {out['loss'][k]:9.5f}  mean reward {out['reward'][k]:.3f}")
    print(f"after {steps} steps: mean reward {out['reward_after']:.3f}; at the median score {out['shipped']:.0%} of the "
          "answers ship")
    return 0


if __name__ == "__main__":
    sys.exit(main(sys.argv[1:]))
