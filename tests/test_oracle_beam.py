"""The oracle of the largest logits, the distillation loss and beam search, pinned by brute force, closed forms and
differences (CPU only)."""

import itertools
import math

import numpy as np
import pytest

from oracle import beam as obeam
from oracle import distill as odist


def rows(n, V, seed, scale=2.0):
    return np.random.default_rng(seed).normal(0, scale, (n, V)).astype(np.float32)


def softmax(z, T):
    e = [math.exp(float(x) / T) for x in z]
    s = math.fsum(e)
    return [x / s for x in e]


def test_top_logits_by_hand():
    z = np.array([[1.0, 3.0, 3.0, -np.inf, 2.0, -0.0, 0.0]], np.float32)
    o = odist.top_logits(z, "f32", np.ones(1, np.float32), 7)
    assert o["ids"].tolist() == [[1, 2, 4, 0, 5, 6, -1]]
    p = softmax([1, 3, 3, -1e300, 2, 0, 0], 1.0)
    assert np.allclose(np.exp(o["logprob"][0, :6]), [p[i] for i in (1, 2, 4, 0, 5, 6)], rtol=1e-13)
    assert o["logprob"][0, 6] == -np.inf and abs(o["lse"][0] - math.log(sum(map(math.exp, (1, 3, 3, 2, 0, 0))))) < 1e-13


def test_top_logits_undefined_rows():
    z = np.zeros((4, 3), np.float32)
    z[0, 1], z[1, 0], z[2] = np.nan, np.inf, -np.inf
    o = odist.top_logits(z, "f32", np.array([1, 1, 1, 0], np.float32), 2)
    assert o["flags"].tolist() == [1, 1, 1, 4] and (o["ids"] == -1).all() and np.isnan(o["logprob"]).all()


def direct_loss(z, T, ids, logq, tail):
    """The definition, in plain Python."""
    p = softmax(z, T)
    entries = [(v, math.exp(x)) for v, x in zip(ids, logq) if x > -math.inf]
    Q = sum(q for _, q in entries)
    if tail == "renorm":
        entries = [(v, q / Q) for v, q in entries]
    l = sum(q * math.log(q / p[v]) for v, q in entries)
    if tail == "rest" and 1 - Q > 0:
        P = sum(p[v] for v, _ in entries)
        l += (1 - Q) * math.log((1 - Q) / (1 - P))
    return l


@pytest.mark.parametrize("tail", ["drop", "renorm", "rest"])
def test_loss_by_definition_and_differences(tail):
    n, V, k = 4, 9, 3
    z, T = rows(n, V, 1), np.array([1.0, 0.5, 2.0, 0.75], np.float32)
    teacher = rows(n, V, 2)
    ids = np.argsort(-teacher, axis=1)[:, :k].astype(np.int32)
    logq = np.array([[math.log(softmax(teacher[r], 1.0)[v]) for v in ids[r]] for r in range(n)], np.float32)
    logq[2, 1] = -np.inf
    w = np.array([0.5, 2.0, 1.0, -0.25], np.float32)
    o = odist.distill_loss(z, "f32", ids, logq, T, w, tail, grad_scale=3.0)
    total = 0.0
    for r in range(n):
        direct = direct_loss(z[r], float(T[r]), ids[r], logq[r].astype(float), tail)
        assert abs(o["token_loss"][r] - direct) < 1e-12
        total += float(w[r]) * direct
        for v in range(V):
            h = 1e-5
            up, down = z[r].astype(float).copy(), z[r].astype(float).copy()
            up[v] += h
            down[v] -= h
            d = (direct_loss(up, float(T[r]), ids[r], logq[r].astype(float), tail)
                 - direct_loss(down, float(T[r]), ids[r], logq[r].astype(float), tail)) / (2 * h)
            assert abs(o["grad"][r, v] - 3.0 * float(w[r]) * d) < 1e-8
    assert abs(o["loss"] - total) < 1e-12


def test_loss_is_zero_at_the_teacher():
    z = rows(3, 20, 5)
    one = np.ones(3, np.float32)
    top = odist.top_logits(z, "f32", one, 5)
    o = odist.distill_loss(z, "f32", top["ids"], top["logprob"], one, one, "rest")
    assert np.abs(o["token_loss"]).max() < 1e-12 and np.abs(o["grad"]).max() < 1e-12
    full = odist.top_logits(z, "f32", one, 20)
    for tail in ("drop", "renorm", "rest"):
        o = odist.distill_loss(z, "f32", full["ids"], full["logprob"], one, one, tail)
        assert np.abs(o["token_loss"]).max() < 1e-12 and np.abs(o["grad"]).max() < 1e-12


def test_loss_readings():
    z = rows(6, 5, 7)
    z[4, 1:] = -np.inf
    ids = np.array([[0, 1], [0, 0], [5, 1], [0, 1], [0, 2], [-1, 7]], np.int32)
    logq = np.log(np.array([[0.5, 0.25], [0.5, 0.25], [0.5, 0.25], [0.5, np.nan], [0.9, 0.0], [0.0, 0.0]], np.float32) + 0)
    one = np.ones(6, np.float32)
    w = one.copy()
    w[0] = 0
    o = odist.distill_loss(z, "f32", ids, logq, one, w, "rest")
    assert o["flags"].tolist() == [16, 2, 2, 1, 0, 0]
    assert (o["grad"][0] == 0).all() and np.isnan(o["grad"][1:4]).all() and math.isnan(o["loss"])
    assert abs(o["token_loss"][4] - 0.9 * math.log(0.9)) < 1e-7  # nothing left beside token 0
    assert o["token_loss"][5] == 0.0 and np.abs(o["grad"][5]).max() < 1e-15  # no entries: the rest is everything
    for tail in ("drop", "renorm"):
        o = odist.distill_loss(z[5:], "f32", ids[5:], logq[5:], one[5:], one[5:], tail)
        assert o["loss"] == 0.0 and (o["grad"] == 0).all()
    gone = z[:1].copy()
    gone[0, 0] = -np.inf
    assert odist.distill_loss(gone, "f32", ids[:1], logq[:1], one[:1], one[:1], "drop")["loss"] == math.inf


def brute(z, T, scores, k, done=None, token=-1):
    n_req, B = scores.shape
    out = []
    for i in range(n_req):
        c = []
        for b in range(B):
            if scores[i, b] == -np.inf:
                continue
            if done is not None and done[i, b]:
                c.append((-float(scores[i, b]), b, 0, 0, token))
                continue
            p = softmax(z[i * B + b], float(T[i * B + b]))
            c += [(-(float(scores[i, b]) + math.log(p[v])), b, -float(z[i * B + b][v]), v, v) for v in range(len(p)) if p[v] > 0]
        out.append([(b, t) for _, b, _, _, t in sorted(c)[:k]])
    return out


@pytest.mark.parametrize("B,k", list(itertools.product((1, 3), (1, 3, 7, 40))))
def test_beam_select_by_brute_force(B, k):
    n_req, V = 3, 11
    z = np.round(rows(n_req * B, V, 10 * B + k), 1)  # ties within a beam
    T = np.full(n_req * B, 0.8, np.float32)
    scores = np.random.default_rng(k).normal(-3, 1, (n_req, B)).astype(np.float32)
    if B > 1:
        scores[1, 1] = -np.inf
    done = np.zeros((n_req, B), bool)
    done[2, 0] = True
    o = obeam.beam_select(z, "f32", T, scores, k, done, 77)
    want = brute(z, T, scores, k, done, 77)
    for i in range(n_req):
        got = [(b, t) for b, t in zip(o["parent"][i], o["token"][i]) if b >= 0]
        assert got == want[i]
        assert (np.diff(o["scores"][i][:len(got)]) <= 0).all()
        assert (o["token"][i][len(got):] == -1).all() and (o["scores"][i][len(got):] == -np.inf).all()


def test_beam_flags():
    z = np.zeros((5, 4), np.float32)
    z[3, 0] = np.nan
    scores = np.array([[np.nan, np.inf, -np.inf, 0.0, 0.0]], np.float32)
    o = obeam.beam_select(z, "f32", np.ones(5, np.float32), scores, 3)
    assert o["flags"].tolist() == [1, 1, 16, 1, 0]
    assert o["parent"].tolist() == [[4, 4, 4]] and o["token"].tolist() == [[0, 1, 2]]


def test_reorder():
    x = np.arange(12).reshape(6, 2)
    assert obeam.reorder(x, [[2, 0, 0], [1, -1, 3]]).tolist() == [[4, 5], [0, 1], [0, 1], [8, 9], [8, 9], [10, 11]]


@pytest.mark.parametrize("shift", [0.0, 1e10, -1e25])
def test_log_probs_of_rows_far_from_zero(shift):
    """Log-probs do not depend on what a row's logits have in common (here all V are equal)."""
    V = 400
    lp, lse, flags = odist.row_logprobs(np.full(V, shift, np.float32), "f32", 1.0)
    assert flags == 0 and np.abs(lp + np.log(V)).max() <= 1e-12
    assert abs(lse - (float(np.float32(shift)) + np.log(V))) <= 1e-15 * (1.0 + abs(shift))
