"""fp64 oracle: a step of beam search, and the reordering of states.

TEST INFRASTRUCTURE ONLY -- see the package docstring. Shares no code with
the HIP library.

Candidates of a request are the tokens of its beams, of score
score[b] + log softmax(z_b / T_b)[v]; the k best come first.

Readings:

R31  Order: larger score, lower beam, then the beam's own tokens (larger raw
     logit, lower index). A token of probability 0 and a beam of score -inf make
     no candidate; an ended beam makes one, itself.
R32  A beam whose score is NaN or +inf, or whose row is undefined, makes none
     and is flagged; the search goes on with the others.
"""

from __future__ import annotations

import numpy as np

from .distill import FLAG_MASKED, row_logprobs
from .features import FLAG_NONFINITE, decode_logits


def candidates(raw, dtype, T, scores, done, done_token, k):
    """Every candidate of every request in order, as (score, beam, token, log-prob), at most k a beam; beams' flags."""
    n_req, B = np.shape(scores)
    out, flags = [], np.zeros(n_req * B, dtype=np.int64)
    for i in range(n_req):
        mine = []
        for b in range(B):
            r, s = i * B + b, float(scores[i][b])
            if not s < np.inf:
                flags[r] = FLAG_NONFINITE
            elif s == -np.inf:
                flags[r] = FLAG_MASKED
            elif done is not None and done[i][b]:
                flags[r] = FLAG_MASKED
                mine.append((s, b, 0, done_token, 0.0))
            else:
                lp, _, flags[r] = row_logprobs(raw[r], dtype, T[r])
                if flags[r]:
                    continue
                z = decode_logits(raw[r], dtype)
                order = np.lexsort((np.arange(len(z)), -z))
                order = order[z[order] > -np.inf][:k]
                mine += [(s + lp[v], b, j, int(v), lp[v]) for j, v in enumerate(order)]
        mine.sort(key=lambda c: (-c[0], c[1], c[2]))
        out.append([(s, b, v, l) for s, b, _, v, l in mine])
    return out, flags


def beam_select(raw, dtype, T, scores, k, done=None, done_token=-1) -> dict:
    lists, flags = candidates(raw, dtype, T, scores, done, done_token, k)
    n_req = len(lists)
    out = {"scores": np.full((n_req, k), -np.inf), "parent": np.full((n_req, k), -1), "token": np.full((n_req, k), -1),
           "logprob": np.full((n_req, k), -np.inf), "flags": flags, "candidates": lists}
    for i, mine in enumerate(lists):
        for j, (s, b, v, l) in enumerate(mine[:k]):
            out["scores"][i, j], out["parent"][i, j], out["token"][i, j], out["logprob"][i, j] = s, b, v, l
    return out


def reorder(rows, parent):
    """rows: [n_req * n_beams, ...]; a new array in the beams' new order."""
    n_req, B = np.shape(parent)
    out = np.array(rows)
    for i in range(n_req):
        for b in range(B):
            p = int(parent[i][b])
            if 0 <= p < B:
                out[i * B + b] = rows[i * B + p]
    return out
