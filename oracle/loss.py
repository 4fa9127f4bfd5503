"""fp64 oracle: the losses over logit rows and their gradients.

TEST INFRASTRUCTURE ONLY -- see the package docstring. Shares no code with
the HIP library.

With u = z / T and l = log softmax(u)[y] per row:

* policy: ratio = exp(l - old), gain = min(ratio A, clip(ratio) A),
  kl = exp(ref - l) - 1 - (ref - l), loss = sum of w (kl_coef kl - gain);
* preference: q = sum over a request's rows of w (l - ref),
  h = beta (q_chosen - q_rejected) - margin, loss = mean over pairs of
  -(1 - s) log sigmoid(h) - s log sigmoid(-h).

A row's gradient in the logits is (dloss/dl) / T (onehot(y) - softmax(u)).

Readings:

R24  A row of weight 0 takes no part: its logits, id and temperature may be
     anything, its outputs and its gradient are 0, and it is flagged MASKED.
R25  A row that counts and is NONFINITE, BAD_TP or BAD_ID (the rules of R1, R3
     and R7) has l = NaN: the loss and the row's gradient are NaN.
R26  At ratio A == clip(ratio) A the gradient goes through the ratio: only a
     strictly smaller clipped product stops it. kl_coef = 0 leaves the KL term
     out also where the KL is infinite (a token of probability 0).
"""

from __future__ import annotations

import math

import numpy as np

from .features import FLAG_BAD_ID, FLAG_BAD_TP, FLAG_NONFINITE, decode_logits, token_features

FLAG_MASKED = 16
FLAG_CLIPPED = 32

_UNDEFINED = FLAG_NONFINITE | FLAG_BAD_TP | FLAG_BAD_ID


def _rows(raw, dtype, ids, T, weight):
    """l, flags and softmax of every row."""
    n = len(ids)
    l, flags = np.zeros(n), np.zeros(n, dtype=np.int64)
    p = [None] * n
    for r in range(n):
        if weight[r] == 0:
            flags[r] = FLAG_MASKED
            continue
        f = token_features(raw[r], dtype, int(ids[r]), float(T[r]))
        flags[r] = f["flags"] & _UNDEFINED
        if flags[r]:
            l[r] = np.nan
            continue
        u = decode_logits(raw[r], dtype) / float(np.float32(T[r]))
        u = u - u.max()
        e = np.exp(u)
        S = math.fsum(e)
        l[r] = u[int(ids[r])] - math.log(S)
        p[r] = e / S
    return l, flags, p


def _gradient(shape, ids, T, l, flags, p, dl):
    g = np.zeros(shape)
    for r in range(shape[0]):
        if flags[r] & FLAG_MASKED:
            continue
        if flags[r] & _UNDEFINED:
            g[r] = np.nan
            continue
        onehot = np.zeros(shape[1])
        onehot[int(ids[r])] = 1.0
        with np.errstate(invalid="ignore"):
            g[r] = 0.0 if dl[r] == 0 else dl[r] / float(np.float32(T[r])) * (onehot - p[r])
    return g


def policy_loss(raw, dtype, ids, T, weight, advantage, old_logprob, ref_logprob=None, clip_low=0.2, clip_high=0.2,
                kl_coef=0.0, grad_scale=1.0) -> dict:
    l, flags, p = _rows(raw, dtype, ids, T, weight)
    n = len(l)
    ratio, kl, dl = np.zeros(n), np.zeros(n), np.zeros(n)
    terms = []
    for r in range(n):
        if flags[r] & FLAG_MASKED:
            continue
        w, A = float(weight[r]), float(advantage[r])
        ratio[r] = math.exp(l[r] - float(old_logprob[r]))
        bounded = min(max(ratio[r], 1.0 - clip_low), 1.0 + clip_high)
        clipped = ratio[r] * A > bounded * A
        if clipped:
            flags[r] |= FLAG_CLIPPED
        d = float(ref_logprob[r]) - l[r] if ref_logprob is not None else 0.0
        kl[r] = math.inf if d == math.inf else math.expm1(d) - d
        beta_kl, beta_rise = (kl_coef * kl[r], kl_coef * math.expm1(d)) if kl_coef else (0.0, 0.0)
        terms.append(w * (beta_kl - (bounded * A if clipped else ratio[r] * A)))
        dl[r] = w * ((0.0 if clipped else -ratio[r] * A) - beta_rise)
    if ref_logprob is None:
        kl[:] = 0.0
    return {"loss": math.fsum(terms) if not any(map(math.isnan, terms)) else math.nan, "logprob": l, "ratio": ratio,
            "kl": kl, "flags": flags, "dl": dl,
            "grad": _gradient((n, np.shape(raw)[1]), ids, T, l, flags, p, dl * grad_scale)}


def preference_loss(raw, dtype, ids, T, weight, offsets, ref_logprob=None, beta=0.1, label_smoothing=0.0, margin=0.0,
                    grad_scale=1.0) -> dict:
    l, flags, p = _rows(raw, dtype, ids, T, weight)
    n, n_pairs = len(l), (len(offsets) - 1) // 2
    q = np.zeros(2 * n_pairs)
    for i in range(2 * n_pairs):
        q[i] = sum(float(weight[r]) * (l[r] - (float(ref_logprob[r]) if ref_logprob is not None else 0.0))
                   for r in range(offsets[i], offsets[i + 1]) if weight[r] != 0)
    h = beta * (q[0::2] - q[1::2]) - margin
    s = label_smoothing
    pair = (1 - s) * np.logaddexp(0.0, -h) + s * np.logaddexp(0.0, h)
    # d/dh: s sigmoid(h) - (1 - s) sigmoid(-h)
    dh = s * np.exp(-np.logaddexp(0.0, -h)) - (1 - s) * np.exp(-np.logaddexp(0.0, h))
    dl = np.zeros(n)
    for i in range(2 * n_pairs):
        for r in range(offsets[i], offsets[i + 1]):
            if weight[r] != 0:
                dl[r] = float(weight[r]) * beta * dh[i // 2] / n_pairs * (1 if i % 2 == 0 else -1)
                if np.isnan(dl[r]) and not flags[r] & _UNDEFINED:
                    p[r] = np.full_like(p[r], np.nan)
    with np.errstate(invalid="ignore"):
        loss = float(np.mean(pair)) if n_pairs else math.nan
    return {"loss": loss, "pair_loss": pair, "pair_logit": h, "seq_logratio": q, "logprob": l, "flags": flags,
            "dl": dl, "grad": _gradient((n, np.shape(raw)[1]), ids, T, l, flags, p, dl * grad_scale)}
