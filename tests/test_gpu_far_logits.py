"""Logits far from zero: masks of large finite values (-1e9 .. the type's lowest one) over whole stretches of a row, and
rows that are far as a whole, for the entry points that sum a row's exps.

Scaled logits of 2^30 and more round by more than an exp can hold; there, two logits that differ are so far apart that
only equal ones count beside the largest. The references are in 64 bits; tolerances as in the operators' own tests."""

import math

import numpy as np
import pytest
import torch

import paper_2608_28726_amd as pr
from oracle import beam as obeam
from oracle import distill as odist
from oracle import loss as oloss
from tests.gpu_common import require_gpu
from tests.test_gpu_beam import compare_select, compare_top
from tests.test_gpu_loss import L_ABS, name_of, near, raw_of

pytestmark = pytest.mark.gpu

TEMPERATURES = (0.5, 0.9, 1.0, 1.45, 1.6, 30.0)
SHAPES = [(400, torch.float32), (400, torch.bfloat16), (33001, torch.bfloat16), (33000, torch.float32),
          (160001, torch.bfloat16)]


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def cuda(x):
    return torch.tensor(np.ascontiguousarray(x), device="cuda")


def far_rows(V, dtype, seed):
    """Logits [n, V], temperatures, and of each row some tokens that are not masked."""
    rng = np.random.default_rng(seed)
    low = torch.finfo(dtype).min
    rows, temps, tokens = [], [], []

    def add(z, T, of):
        rows.append(z)
        temps.append(T)
        tokens.append(rng.choice(of, 6, replace=len(of) < 6))

    for T in TEMPERATURES:
        for mask in (-1e9, -1e10, -3e10, -1e30, -3.3e38, low):
            z = rng.normal(0, 2, V)
            free = max(8, V // 10)
            kind = len(rows) % 3
            if kind == 0:  # what is left comes last
                z[:V - free] = mask
                of = np.arange(V - free, V)
            elif kind == 1:  # first
                z[free:] = mask
                of = np.arange(free)
            else:  # a few in one place, two masks
                z[:] = mask
                z[:V // 2] = -2e9
                of = np.arange(V // 2 - 4, V // 2 + 4)
                z[of] = rng.normal(0, 2, 8)
            add(z, T, of)
        # far as a whole: the type keeps steps of the distance, so that most are equal
        for shift in (1e9, -1e9, 1e10, -1e10, 3e12, -1e13, 1e25, -1e25):
            add(rng.normal(0, 2, V) + shift, T, np.arange(V))
        # near 2^30 of scaled logits, on both sides
        edge = 2.0 ** 30 * math.log(2.0) * T
        add(np.where(rng.random(V) < 0.9, edge * 0.999, edge), T, np.arange(V))
        add(np.where(rng.random(V) < 0.5, -edge, -edge * 1.001), T, np.arange(V))
    logits = torch.tensor(np.stack(rows)).to(dtype)
    return logits, np.array(temps, np.float32), np.stack(tokens).astype(np.int32)


def batches(n):
    """Which rows of the n a call takes: a few (spread over the device), and all four times over."""
    yield np.arange(0, n, max(1, n // 7))
    yield np.arange(n // 2, n // 2 + 5)
    yield np.tile(np.arange(n), 4)


def log_softmax64(logits, T):
    u = logits.double().numpy() / T[:, None].astype(np.float64)
    m = u.max(1, keepdims=True)
    return u - m - np.log(np.exp(u - m).sum(1, keepdims=True))


@pytest.mark.parametrize("V,dtype", SHAPES)
def test_top_logits(V, dtype):
    logits, T, _ = far_rows(V, dtype, V)
    for k in (5, 70):
        o = odist.top_logits(raw_of(logits), name_of(dtype), T, k)
        assert not o["flags"].any()
        for at in batches(len(T)):
            print("case", V, dtype, k, len(at), flush=True)
            compare_top(pr.top_logits(logits[at].cuda(), k, cuda(T[at])), {name: x[at] for name, x in o.items()})


@pytest.mark.parametrize("V,dtype", SHAPES[:4])
def test_beam_select(V, dtype):
    logits, T, _ = far_rows(V, dtype, V + 1)
    B = 3
    for at in batches(len(T)):
        at = at[:len(at) // B * B][:60]
        scores = np.random.default_rng(V).normal(-5, 1, (len(at) // B, B)).astype(np.float32)
        o = obeam.beam_select(raw_of(logits[at]), name_of(dtype), T[at], scores, 5)
        compare_select(pr.beam_select(logits[at].cuda(), cuda(scores), cuda(T[at]), 5), o)


@pytest.mark.parametrize("V,dtype", SHAPES)
def test_policy_loss(V, dtype):
    logits, T, tokens = far_rows(V, dtype, V + 2)
    lp = log_softmax64(logits, T)
    n = len(T)
    ids = tokens[:, 0].copy()
    A = np.linspace(-1, 1.5, n).astype(np.float32)
    ids[::5] = np.arange(0, n, 5) % V  # any token, masked ones among them: their ratio is left out of the loss
    A[::5] = 0.0
    old = lp[np.arange(n), ids].astype(np.float32)
    w = np.linspace(0.5, 2, n).astype(np.float32)
    o = oloss.policy_loss(raw_of(logits), name_of(dtype), ids, T, w, A, old)
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    for at in batches(n):
        for grad in (True, False):
            print("case", V, dtype, len(at), grad, flush=True)
            g = pr.policy_loss(logits[at].cuda(), cuda(ids[at]), cuda(T[at]), cuda(w[at]), cuda(A[at]), cuda(old[at]), grad=grad)
            torch.cuda.synchronize()
            assert np.array_equal(g["flags"].cpu().numpy() & 7, o["flags"][at] & 7)
            near("logprob", g["logprob"].cpu().numpy(), lp[np.arange(n), ids][at], L_ABS)
            if grad:
                # The ratio is off by the log-prob's error, the softmax by that of its sum: 4e-6 of the coefficient each.
                coef = np.abs(o["dl"] / T)[at][:, None]
                near("grad", g["grad"].float().cpu().numpy(), o["grad"][at], 1e-5 * coef + 1e-38, half * 1.01 + 1e-5)


@pytest.mark.parametrize("V,dtype", SHAPES[:4])
def test_preference_loss(V, dtype):
    logits, T, tokens = far_rows(V, dtype, V + 3)
    lp = log_softmax64(logits, T)
    n = len(T) // 2 * 2
    ids = tokens[:n, 0]
    l = lp[np.arange(n), ids]
    ref = (l - 0.3).astype(np.float32)
    w = np.linspace(0.5, 2, n).astype(np.float32)
    offsets = np.arange(0, n + 1, 1, dtype=np.int32)
    for rows in (n, 6):
        o = oloss.preference_loss(raw_of(logits[:rows]), name_of(dtype), ids[:rows], T[:rows], w[:rows], offsets[:rows + 1],
                                  ref[:rows])
        g = pr.preference_loss(logits[:rows].cuda(), cuda(ids[:rows]), cuda(T[:rows]), cuda(w[:rows]),
                               cuda(offsets[:rows + 1]), cuda(ref[:rows]))
        torch.cuda.synchronize()
        assert not g["flags"].any()
        near("logprob", g["logprob"].cpu().numpy(), l[:rows], L_ABS)
        half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
        coef = np.abs(o["dl"] / T[:rows])[:, None]
        near("grad", g["grad"].float().cpu().numpy(), o["grad"], 1e-5 * coef + 1e-38, half * 1.01 + 1e-5)


def distill64(lp, ids, lq, T, w, tail):
    """Token losses and gradients in 64 bits, the rest's shares relative to its own sum."""
    n, V = lp.shape
    loss, grad = np.zeros(n), np.zeros((n, V))
    for r in range(n):
        there = lq[r] > -np.inf
        v, x = ids[r][there], lq[r][there].astype(np.float64)
        q = np.exp(x)
        Q = q.sum()
        mine = np.zeros(V, bool)
        mine[v] = True
        others = lp[r][~mine]
        lo = others.max() + np.log(np.exp(others - others.max()).sum())
        share = np.where(mine, 0.0, np.exp(np.minimum(lp[r] - lo, 0.0)))
        P = np.exp(lp[r][mine]).sum()
        rq = max(0.0, 1.0 - Q) if tail == "rest" else 0.0
        scale = 1.0 / Q if tail == "renorm" else 1.0
        total = Q * scale
        loss[r] = (q * scale * (x + math.log(scale) - lp[r][v])).sum() + (rq * (math.log(rq) - lo) if rq > 0 else 0.0)
        g = total * np.exp(lp[r]) - rq * P * share
        dense = np.zeros(V)
        dense[v] = q * scale
        g[mine] = (total + rq) * np.exp(lp[r])[mine] - dense[mine]
        grad[r] = g * float(w[r]) / float(T[r])
    return loss, grad


@pytest.mark.parametrize("V,dtype", SHAPES)
@pytest.mark.parametrize("tail", ["rest", "drop", "renorm"])
def test_distill_loss(V, dtype, tail):
    logits, T, tokens = far_rows(V, dtype, V + 4)
    n = len(T)
    rng = np.random.default_rng(V)
    lp = log_softmax64(logits, T)
    ids = np.tile(np.arange(6), (n, 1)).astype(np.int32)
    for r in range(n):
        mine = np.unique(tokens[r])[:5]
        ids[r, :len(mine)] = mine
        ids[r, len(mine):] = np.setdiff1d(np.arange(12), mine)[:6 - len(mine)]  # any others, masked ones among them
    lq = np.log(rng.dirichlet(np.ones(6), n) * 0.9).astype(np.float32)
    lq[:, 5] = -np.inf
    w = np.linspace(0.5, 2, n).astype(np.float32)
    loss, grad = distill64(lp, ids, lq, T, w, tail)
    half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    for at in batches(n):
        for want_grad in (True, False):
            print("case", V, dtype, tail, len(at), want_grad, flush=True)
            g = pr.distill_loss(logits[at].cuda(), cuda(ids[at]), cuda(lq[at]), cuda(T[at]), cuda(w[at]), tail, grad=want_grad)
            torch.cuda.synchronize()
            assert not g["flags"].any()
            with np.errstate(over="ignore"):
                want = np.where(np.isinf(loss[at].astype(np.float32)), np.inf, loss[at])
            near("token_loss", g["token_loss"].cpu().numpy(), want, 2 * L_ABS)
            if want_grad:
                near("grad", g["grad"].float().cpu().numpy(), grad[at], 6e-6 * (w / T)[at][:, None] + 1e-38,
                     half * 1.01 + 2.0 ** -22)
