"""The verifier's features, sequence, draws and streamed tokens of rows with masks of large finite values, and of rows far
from zero (the rows of test_gpu_far_logits), against the oracle. Tolerances: those of the features' own tests."""

import numpy as np
import pytest
import torch

import oracle
import paper_2608_28726_amd as pr
from oracle import sequence as oseq
from tests.gpu_common import compare_features, require_gpu
from tests.helpers import assert_floats
from tests.test_gpu_far_logits import SHAPES, cuda, far_rows, log_softmax64
from tests.test_gpu_loss import name_of, raw_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def batches(n, V):
    """Rows of a call: a few (several workgroups a row), all, and so many that each size of workgroup takes them."""
    yield np.arange(0, n, 12)
    yield np.arange(n)
    yield np.tile(np.arange(n), 4)
    if V < 40000:
        yield np.tile(np.arange(n), 13)


def expected(logits, ids, T, P=None):
    o = oracle.token_features_batch(raw_of(logits), name_of(logits.dtype), ids, T, P)
    o = {k: np.asarray(v) for k, v in o.items()}
    assert not (o["flags"] & 7).any()
    # The oracle's log-prob is u_y - lse, which loses log S where u is 1e10 and more. maxprob is 1 / S.
    u = logits.double().numpy() / T[:, None].astype(np.float64)
    there = np.isfinite(o["logprob"])
    exact = u[np.arange(len(T)), ids] - u.max(1) + np.log(o["maxprob"])
    with np.errstate(over="ignore"):
        exact = np.where(np.isinf(exact.astype(np.float32)), -np.inf, exact)
    o["logprob"] = np.where(there, exact, o["logprob"])
    return o


def some_ids(logits, tokens):
    """Tokens that are not masked, and in every fifth row any."""
    ids = tokens[:, 0].copy()
    ids[::5] = (np.arange(len(ids)) * 37 % logits.shape[1])[::5]
    return ids


@pytest.mark.parametrize("V,dtype", SHAPES)
@pytest.mark.parametrize("top_p", [None, 0.9, 1.0])
def test_token_features(V, dtype, top_p):
    logits, T, tokens = far_rows(V, dtype, V + 10)
    ids = some_ids(logits, tokens)
    P = None if top_p is None else np.full(len(T), top_p, np.float32)
    o = expected(logits, ids, T, P)
    for at in batches(len(T), V):
        print("case", V, dtype, top_p, len(at), flush=True)
        f = pr.token_features(logits[at].cuda(), cuda(ids[at]), cuda(T[at]), None if P is None else cuda(P[at]))
        torch.cuda.synchronize()
        compare_features({k: v.cpu().numpy() for k, v in f.items()}, {k: v[at] for k, v in o.items()})


@pytest.mark.parametrize("V,dtype", SHAPES)
@pytest.mark.parametrize("top_p", [None, 0.9])
def test_sequence(V, dtype, top_p):
    """Rows with fewer tokens left than the top-K entropy takes are among them (8 of 20)."""
    logits, T, tokens = far_rows(V, dtype, V + 11)
    ids = tokens[:, 0]
    P = None if top_p is None else np.full(len(T), top_p, np.float32)
    o = expected(logits, ids, T, P)
    H = oseq.topk_entropy_batch(raw_of(logits), name_of(dtype), T, P)
    for at in batches(len(T), V):
        print("case", V, dtype, top_p, len(at), flush=True)
        offsets = np.array([0, len(at)], np.int32)
        X = pr.feature_sequence(logits[at].cuda(), cuda(ids[at]), cuda(T[at]), cuda(offsets),
                                None if P is None else cuda(P[at]))
        torch.cuda.synchronize()
        X = X.cpu().numpy()
        assert_floats("logprob", X[:, 0], o["logprob"][at])
        assert_floats("maxprob", X[:, 1], o["maxprob"][at])
        assert_floats("entropy", -X[:, 2], H[at], mask=~o["ambiguous"][at])


@pytest.mark.parametrize("V,dtype", SHAPES)
@pytest.mark.parametrize("with_sequence", [False, True])
def test_draws(V, dtype, with_sequence):
    """A token is drawn from every row, none that is masked, and its features are the row's; where all logits are equal
    the draws spread over the row."""
    logits, T, _ = far_rows(V, dtype, V + 12)
    logits[0], logits[1] = -1e10, 3e12  # all equal
    lp = log_softmax64(logits, T)
    for at in batches(len(T), V):
        print("case", V, dtype, with_sequence, len(at), flush=True)
        offsets = cuda(np.array([0, len(at)], np.int32)) if with_sequence else None
        ids, f, _ = pr.sample_features(logits[at].cuda(), cuda(T[at]), 5, offsets=offsets)
        torch.cuda.synchronize()
        y = ids.cpu().numpy()
        assert (y >= 0).all()
        drawn = lp[at, y]
        assert drawn.min() > -60.0  # e^-60: no mask, and nothing that is never drawn
        assert_floats("logprob", f["logprob"].cpu().numpy(), drawn)
        assert not (f["flags"].cpu().numpy() & 7).any()
    logits = torch.full((600, V), -1e10).to(dtype)
    ids, _, _ = pr.sample_features(logits.cuda(), torch.ones(600, device="cuda"), 6)
    y = np.sort(ids.cpu().numpy()) / V
    # Kolmogorov's distance of 600 uniform draws is beyond 0.1 once in 2e5 runs; the draw is fixed by its seed.
    assert np.abs(y - (np.arange(600) + 0.5) / 600).max() < 0.1


@pytest.mark.parametrize("V,dtype", SHAPES[:4])
@pytest.mark.parametrize("max_len", [0, 4])
def test_streamed_tokens(V, dtype, max_len):
    logits, T, tokens = far_rows(V, dtype, V + 13)
    n = len(T)
    ids = tokens[:, 0]
    o = expected(logits, ids, T)
    state = pr.StreamState(n, max_len)
    slots = torch.arange(n, dtype=torch.int32, device="cuda")
    f = state.step(logits.cuda(), slots, cuda(ids), cuda(T), want_features=True)
    few = np.arange(0, n, 12)
    state.step(logits[few].cuda(), cuda(few.astype(np.int32)), cuda(ids[few]), cuda(T[few]))
    score = state.finish(slots, 0.0)["score"]
    torch.cuda.synchronize()
    compare_features({k: v.cpu().numpy() for k, v in f.items()}, o)
    assert_floats("score", score.cpu().numpy(), o["maxprob"])  # the mean of maxprob, which the second step leaves
    state.close()


@pytest.mark.parametrize("n", [6, 300, 2100])
@pytest.mark.parametrize("low,high", [(3 * 2.0 ** 39, 3 * 2.0 ** 40), (-3 * 2.0 ** 41, -3 * 2.0 ** 40), (-3e38, -1e10), (1e9, 3e12)])
def test_the_one_token_that_is_larger_is_drawn(n, low, high):
    """Rows of one far value but for a larger one, which has all the probability (pairs a power of two apart among them,
    whose references look alike)."""
    V = 33000
    rng = np.random.default_rng(n)
    at = rng.integers(0, V, n)
    at[:3] = 0, V // 2, V - 1
    z = torch.full((n, V), low, device="cuda")
    z[torch.arange(n), cuda(at)] = high
    ids, f, _ = pr.sample_features(z, torch.ones(n, device="cuda"), 9)
    torch.cuda.synchronize()
    assert np.array_equal(ids.cpu().numpy(), at)
    assert (f["logprob"] == 0).all() and (f["maxprob"] == 1).all()
