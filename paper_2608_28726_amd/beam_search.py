"""Beam search over a model's logit rows, with the verifier watching every beam.

One step of the search is four calls: the best continuations of each request's
beams (:func:`beam_select`), the beams' states put into their order
(:func:`beam_reorder`), the verifier's state of each beam likewise
(:meth:`StreamState.reorder`), and the chosen tokens' features
(:meth:`StreamState.step`). The answers can then be routed like any others.

    python -m paper_2608_28726_amd.beam_search [requests] [beams] [length]

decodes seeded synthetic contexts with an output layer and routes the best
answer of each request.
"""

from __future__ import annotations

import sys

import torch

import paper_2608_28726_amd as pr


def beam_search(next_logits, n_req: int, n_beams: int, length: int, temperature: float = 1.0, end: int | None = None,
                states=(), stream: pr.StreamState | None = None, slots: torch.Tensor | None = None,
                device="cuda") -> dict:
    """The ``n_beams`` best answers of each request, of ``length`` tokens or up to the token ``end``.

    ``next_logits(t, tokens)`` returns the logit rows [n_req * n_beams, V] of
    step t; ``tokens`` (int32 [n_req * n_beams], None at step 0) are those that
    the beams were continued with, -1 for beams that have ended or do not exist. ``states``:
    tensors that belong to the beams (:func:`beam_reorder`), reordered in place
    before the next step. ``stream`` and ``slots`` (int32 [n_req, n_beams]):
    the verifier's state and each beam's slot in it; the rows that
    ``next_logits`` returned are then overwritten.

    Returns a dict with ``tokens`` (int32 [n_req, n_beams, length], best beam
    first, -1 after the end), ``scores`` (float32 [n_req, n_beams], sums of
    log-probs) and ``done`` (bool, whether a beam reached ``end``). A beam that
    does not exist (there were fewer candidates) has a score of -inf and no tokens, and its slot is empty.
    """
    n = n_req * n_beams
    scores = torch.full((n_req, n_beams), -torch.inf, dtype=torch.float32, device=device)
    scores[:, 0] = 0.0  # one beam to begin with
    tokens = torch.full((n, length), -1, dtype=torch.int32, device=device)
    done = torch.zeros(n_req, n_beams, dtype=torch.bool, device=device)
    token = None
    for t in range(length):
        logits = next_logits(t, token)
        best = pr.beam_select(logits, scores, temperature, done=done if end is not None else None)
        scores, parent, token = best["scores"], best["parent"], best["token"].view(-1)
        moved = [tokens, done.view(-1), *states]
        if stream is not None:
            moved.append(logits)  # each beam's row is now the one that its token was chosen from
            stream.reorder(slots, parent)
        pr.beam_reorder(moved, parent)
        if stream is not None:
            # Ended beams and beams that do not exist have no token: no slot changes.
            stream.step(logits, torch.where(token.view(n_req, n_beams) < 0, -1, slots).view(-1), token, temperature)
        tokens[:, t] = token
        if end is not None:
            done |= (token == end).view(n_req, n_beams)
    there = scores > -torch.inf
    if stream is not None:
        # What a beam had seen before it ceased to exist is no answer's.
        stream.reset(torch.where(there, -1, slots).view(-1))
    tokens = torch.where(there[..., None], tokens.view(n_req, n_beams, length), -1)
    return {"tokens": tokens, "scores": scores, "done": done & there}


class Contexts:
    """Hidden states that follow the tokens: h' = (h + embedding of the token) / sqrt 2, kept for every step."""

    def __init__(self, hidden: torch.Tensor, vocab: int, n_beams: int, length: int, seed: int):
        g = torch.Generator(device=hidden.device)
        g.manual_seed(seed)
        width = hidden.shape[1]
        self.embedding = torch.empty(vocab, width, dtype=torch.float32, device=hidden.device).normal_(generator=g).bfloat16()
        self.hidden = hidden.repeat_interleave(n_beams, 0)
        self.seen = torch.zeros(self.hidden.shape[0], length, width, dtype=hidden.dtype, device=hidden.device)

    def step(self, t: int, tokens) -> torch.Tensor:
        if tokens is not None:
            move = (self.hidden + self.embedding[tokens.clamp(min=0).long()]) * 0.5 ** 0.5
            self.hidden.copy_(torch.where((tokens >= 0)[:, None], move, self.hidden))
        self.seen[:, t] = self.hidden
        return self.hidden

    @property
    def states(self):
        return [self.hidden, self.seen]


def search(layer, hidden: torch.Tensor, vocab: int, n_beams: int, length: int, seed: int, temperature: float = 1.0,
           end: int | None = None) -> dict:
    """Beam search of an output layer (``layer(hidden)`` gives logit rows) from each of the hidden states. Besides what
    :func:`beam_search` returns: ``contexts`` [n_req, n_beams, length, width], and of every beam the verifier's summary
    ``confidence`` [n_req, n_beams], NaN where there is no beam (no such answer ships)."""
    n_req = hidden.shape[0]
    contexts = Contexts(hidden, vocab, n_beams, length, seed)
    stream = pr.StreamState(n_req * n_beams, length)
    slots = torch.arange(n_req * n_beams, dtype=torch.int32, device=hidden.device)
    out = beam_search(lambda t, tokens: layer(contexts.step(t, tokens)), n_req, n_beams, length, temperature, end,
                      contexts.states, stream, slots.view(n_req, n_beams), hidden.device)
    out["confidence"] = stream.finish(slots, 0.0)["score"].view(n_req, n_beams)
    stream.close()
    out["contexts"] = contexts.seen.view(n_req, n_beams, length, -1)
    return out


def main(argv) -> int:
    requests, beams, length = [int(v) for v in argv] + [16, 4, 12][len(argv):]
    vocab, width, device = 32000, 256, "cuda"
    g = torch.Generator(device=device)
    g.manual_seed(1)
    weight = torch.empty(vocab, width, dtype=torch.float32, device=device).normal_(std=2.0 * width ** -0.5, generator=g)
    weight = weight.bfloat16()
    hidden = torch.empty(requests, width, dtype=torch.float32, device=device).normal_(generator=g).bfloat16()
    out = search(lambda h: h @ weight.t(), hidden, vocab, beams, length, seed=2)
    best = out["confidence"][:, 0].contiguous()
    tau, _ = pr.calibrate_threshold(best, 0.5)
    ship, n_ship = pr.route(best, float(tau))
    for i in range(min(requests, 8)):
        print(f"request {i:3d}  score {out['scores'][i, 0]:8.3f}  confidence {best[i]:.4f}  "
              f"{'ships' if ship[i] else 'escalates'}  {out['tokens'][i, 0].tolist()}")
    print(f"{int(n_ship)} of {requests} answers ship")
    return 0


if __name__ == "__main__":
    sys.exit(main(sys.argv[1:]))
