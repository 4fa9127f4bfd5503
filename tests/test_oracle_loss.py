"""The oracle's losses against closed forms, differences and autograd in
float64. CPU only."""

import math

import numpy as np
import pytest
import torch

from oracle import loss as oloss


def batch(seed, n=9, V=13):
    rng = np.random.default_rng(seed)
    z = rng.normal(0, 2, (n, V)).astype(np.float32)
    ids = rng.integers(0, V, n)
    T = rng.uniform(0.5, 1.5, n).astype(np.float32)
    w = rng.uniform(0.2, 1.0, n).astype(np.float32)
    w[3] = 0.0
    return rng, z, ids, T, w


def logprobs(z, ids, T):
    u = torch.as_tensor(z, dtype=torch.float64) / torch.as_tensor(T, dtype=torch.float64)[:, None]
    return torch.log_softmax(u, 1).gather(1, torch.as_tensor(ids)[:, None])[:, 0]


def policy_torch(z, ids, T, w, A, old, ref, lo, hi, beta):
    l = logprobs(z, ids, T)
    ratio = torch.exp(l - torch.as_tensor(old))
    A = torch.as_tensor(A)
    gain = torch.minimum(ratio * A, ratio.clamp(1 - lo, 1 + hi) * A)
    kl = torch.exp(torch.as_tensor(ref) - l) - 1 - (torch.as_tensor(ref) - l)
    return (torch.as_tensor(w) * (beta * kl - gain)).sum()


def preference_torch(z, ids, T, w, off, ref, beta, s, margin):
    t = torch.as_tensor(w) * (logprobs(z, ids, T) - torch.as_tensor(ref))
    q = torch.stack([t[off[i]:off[i + 1]].sum() for i in range(len(off) - 1)])
    h = beta * (q[0::2] - q[1::2]) - margin
    return (-(1 - s) * torch.nn.functional.logsigmoid(h) - s * torch.nn.functional.logsigmoid(-h)).mean()


@pytest.mark.parametrize("seed", range(4))
def test_policy_gradient(seed):
    rng, z, ids, T, w = batch(seed)
    n = len(ids)
    l = logprobs(z, ids, T).numpy()
    A, old, ref = rng.normal(0, 1, n), l + rng.normal(0, 0.4, n), l + rng.normal(0, 0.5, n)
    args = (ids, T.astype(np.float64), w.astype(np.float64), A, old, ref, 0.2, 0.3, 0.1)
    o = oloss.policy_loss(z, "f32", ids, T, w, A, old, ref, 0.2, 0.3, 0.1)
    zt = torch.tensor(z, dtype=torch.float64, requires_grad=True)
    loss = policy_torch(zt, *args)
    loss.backward()
    assert abs(o["loss"] - float(loss.detach())) < 1e-12
    assert np.abs(o["grad"] - zt.grad.numpy()).max() < 1e-12
    assert (o["grad"][3] == 0).all() and o["flags"][3] == oloss.FLAG_MASKED
    # central differences, away from the clip's corners
    e = 1e-6
    for r, v in ((0, 2), (5, int(ids[5])), (8, 12)):
        up, down = z.astype(np.float64), z.astype(np.float64)
        up[r, v] += e
        down[r, v] -= e
        num = (float(policy_torch(up, *args)) - float(policy_torch(down, *args))) / (2 * e)
        assert abs(num - o["grad"][r, v]) < 1e-7


@pytest.mark.parametrize("s,margin,use_ref", [(0.0, 0.0, True), (0.1, 0.0, True), (0.0, 0.5, False), (1.0, 0.0, True)])
def test_preference_gradient(s, margin, use_ref):
    rng, z, ids, T, w = batch(7)
    off = [0, 2, 5, 5, 9]  # an empty chosen request
    l = logprobs(z, ids, T).numpy()
    ref = l + rng.normal(0, 0.5, len(ids)) if use_ref else None
    o = oloss.preference_loss(z, "f32", ids, T, w, off, ref, 0.4, s, margin)
    zt = torch.tensor(z, dtype=torch.float64, requires_grad=True)
    args = (ids, T.astype(np.float64), w.astype(np.float64), off, ref if use_ref else np.zeros(len(ids)), 0.4, s, margin)
    loss = preference_torch(zt, *args)
    loss.backward()
    assert abs(o["loss"] - float(loss.detach())) < 1e-12
    assert np.abs(o["grad"] - zt.grad.numpy()).max() < 1e-12
    e = 1e-6
    for r, v in ((0, 2), (6, int(ids[6]))):
        up, down = z.astype(np.float64), z.astype(np.float64)
        up[r, v] += e
        down[r, v] -= e
        num = (float(preference_torch(up, *args)) - float(preference_torch(down, *args))) / (2 * e)
        assert abs(num - o["grad"][r, v]) < 1e-8


def test_closed_forms():
    z = np.zeros((2, 4), np.float32)
    # Uniform rows at the old policy: ratio 1, gain A, gradient -A w (onehot - 1/4) / T.
    o = oloss.policy_loss(z, "f32", [1, 2], [2.0, 1.0], [1.0, 0.5], [3.0, -2.0], [-math.log(4)] * 2)
    assert abs(o["loss"] - (-3.0 + 1.0)) < 1e-15 and np.allclose(o["logprob"], -math.log(4), atol=1e-15)
    assert np.allclose(o["grad"], [[0.375, -1.125, 0.375, 0.375], [-0.25, -0.25, 0.75, -0.25]], atol=1e-15)
    # Past the clip on the side that gains: no gradient; on the other side: the ratio's own.
    o = oloss.policy_loss(z, "f32", [0, 0], [1.0, 1.0], [1.0, 1.0], [1.0, -1.0], [-math.log(4) - 1.0] * 2)
    assert (o["grad"][0] == 0).all() and o["flags"].tolist() == [oloss.FLAG_CLIPPED, 0]
    assert abs(o["grad"][1, 0] - math.e * 0.75) < 1e-14
    # Equal answers: h = 0, loss log 2, slope beta / 2.
    o = oloss.preference_loss(z, "f32", [0, 0], [1.0, 1.0], [1.0, 1.0], [0, 1, 2], None, 0.1)
    assert abs(o["loss"] - math.log(2)) < 1e-15 and abs(o["dl"][0] + 0.05) < 1e-16 and abs(o["dl"][1] - 0.05) < 1e-16


def test_undefined_rows():
    z = np.zeros((3, 5), np.float32)
    z[0, 2] = np.nan
    o = oloss.policy_loss(z, "f32", [0, 9, 1], [1.0, 1.0, 1.0], [1.0, 1.0, 1.0], [1.0] * 3, [-1.0] * 3)
    assert math.isnan(o["loss"]) and np.isnan(o["grad"][:2]).all() and np.isfinite(o["grad"][2]).all()
    o = oloss.policy_loss(z, "f32", [0, 9, 1], [1.0, 1.0, 1.0], [0.0, 0.0, 1.0], [1.0] * 3, [-1.0] * 3)
    assert math.isfinite(o["loss"]) and (o["grad"][:2] == 0).all()


def test_no_kl_term_without_a_coefficient():
    """kl_coef = 0: loss and gradient are those without a reference, also at a token of probability 0."""
    z = np.zeros((2, 5), np.float32)
    z[1, 2] = -np.inf
    ids, T, w, A, old = [2, 2], np.ones(2, np.float32), np.ones(2), np.ones(2), np.full(2, -1.0)
    plain = oloss.policy_loss(z, "f32", ids, T, w, A, old)
    o = oloss.policy_loss(z, "f32", ids, T, w, A, old, np.full(2, -1.0))
    assert o["kl"][1] == math.inf and o["kl"][0] > 0
    assert o["loss"] == plain["loss"] and np.array_equal(o["grad"], plain["grad"])
    assert math.isinf(oloss.policy_loss(z, "f32", ids, T, w, A, old, np.full(2, -1.0), kl_coef=0.1)["loss"])
