"""fp64 oracle: a row's largest logits, and the loss of a student's rows against a teacher's log-probs.

TEST INFRASTRUCTURE ONLY -- see the package docstring. Shares no code with
the HIP library.

With u = z / T, p = softmax(u) and a row's entries (v_i, log q_i), Q = sum q_i:

* drop: l = sum of q_i (log q_i - log p_{v_i});
* renorm: the same with q_i / Q;
* rest: drop + r_q (log r_q - log r_p), r_q = max(0, 1 - Q), r_p the sum of p
  over all other tokens;

loss = sum of w l; a row's gradient in the logits is w / T dl/du.

Readings:

R28  A token of probability 0 (logit -inf) is not among a row's largest: the
     rest of a shorter list is id -1, log-prob -inf. Such entries are none in the loss.
R29  The rest is no term where r_p is 0 (no other token is left). RENORM of a
     row without entries (or of probability 0 in all) is 0, as its gradient.
R30  Entries that count must have ids in [0, V), all different (else BAD_ID), and
     log-probs below +inf (else NONFINITE): such a row is NaN like those of R25.
"""

from __future__ import annotations

import math

import numpy as np

from .features import FLAG_BAD_ID, FLAG_BAD_TP, FLAG_NONFINITE, decode_logits, token_features

FLAG_MASKED = 16


def row_logprobs(raw, dtype, T):
    """log softmax(z / T), the log sum of exps and the flags of a row."""
    flags = int(token_features(raw, dtype, 0, float(T))["flags"]) & (FLAG_NONFINITE | FLAG_BAD_TP)
    if flags:
        return None, math.nan, flags
    u = decode_logits(raw, dtype).astype(np.float64) / float(np.float32(T))
    m = u.max()
    rest = math.log(math.fsum(np.exp(u - m)))
    return (u - m) - rest, m + rest, 0


def top_logits(raw, dtype, T, k) -> dict:
    n = len(T)
    ids, logp, lse, flags = np.full((n, k), -1), np.full((n, k), -np.inf), np.zeros(n), np.zeros(n, dtype=np.int64)
    for r in range(n):
        lp, lse[r], flags[r] = row_logprobs(raw[r], dtype, T[r])
        if flags[r]:
            logp[r] = np.nan
            continue
        z = decode_logits(raw[r], dtype)
        order = np.lexsort((np.arange(len(z)), -z))
        order = order[z[order] > -np.inf][:k]
        ids[r, :len(order)] = order
        logp[r, :len(order)] = lp[order]
    return {"ids": ids, "logprob": logp, "lse": lse, "flags": flags}


def distill_loss(raw, dtype, ids, logq, T, weight, tail="rest", grad_scale=1.0) -> dict:
    n, V = np.shape(raw)
    loss, mass, flags = np.zeros(n), np.zeros(n), np.zeros(n, dtype=np.int64)
    grad, dl = np.zeros((n, V)), np.zeros(n)
    terms = []
    for r in range(n):
        if weight[r] == 0:
            flags[r] = FLAG_MASKED
            continue
        lp, lse, flags[r] = row_logprobs(raw[r], dtype, T[r])
        entries = [(int(v), float(x)) for v, x in zip(ids[r], logq[r]) if not x == -np.inf]
        seen = [v for v, _ in entries]
        if any(not x < math.inf for _, x in entries):
            flags[r] |= FLAG_NONFINITE
        if any(v < 0 or v >= V for v in seen) or len(set(seen)) < len(seen):
            flags[r] |= FLAG_BAD_ID
        if flags[r]:
            loss[r] = mass[r] = np.nan
            grad[r] = np.nan
            terms.append(np.nan)
            continue
        Q = math.fsum(math.exp(x) for _, x in entries)
        mine = np.zeros(V, dtype=bool)
        mine[seen] = True
        p = np.exp(lp)
        rest = math.fsum(p[~mine])
        dl[r] = float(weight[r]) / float(np.float32(T[r])) * grad_scale
        logQ = math.log(Q) if tail == "renorm" and Q > 0 else 0.0
        if tail == "renorm" and not Q > 0:
            entries = []
        q = np.zeros(V)
        for v, x in entries:
            q[v] = math.exp(x - logQ)
            if q[v] > 0:
                loss[r] += q[v] * (x - logQ - lp[v])
        Qn = (1.0 if entries and Q > 0 else 0.0) if tail == "renorm" else Q
        rq = max(0.0, 1.0 - Q) if tail == "rest" and (lp[~mine] > -np.inf).any() else 0.0
        inside, outside = Qn + rq, np.full(V, Qn)
        if rq > 0:
            hi = lp[~mine].max()
            log_rest = hi + math.log(math.fsum(np.exp(lp[~mine] - hi)))
            loss[r] += rq * (math.log(rq) - log_rest)
            outside = Qn - rq * math.fsum(p[mine]) * np.exp(-log_rest)
        g = np.where(mine, inside * p - q, outside * p)
        mass[r] = math.fsum(p[mine])
        grad[r] = g * dl[r]
        terms.append(float(weight[r]) * loss[r])
    total = sum(terms) if any(map(math.isnan, terms)) or any(map(math.isinf, terms)) else math.fsum(terms)
    return {"loss": total, "token_loss": loss, "mass": mass, "flags": flags, "coef": dl, "grad": grad}
