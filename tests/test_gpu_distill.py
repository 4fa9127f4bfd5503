"""The distillation loss and its gradient: HIP path vs the fp64 oracle.

Tolerances. As for the policy loss, a log of a row's sum of exps (over all its
tokens, or over those that are no entry's) is within 2e-6, L, of the exact one.
  l = cross + Q lse + r_q (log r_q - (rest - lse)): (Q + 2 r_q) L, at most 2 L max(1, Q), besides 2^-24 of it.
  P = exp(log sum over the entries' tokens - lse): 2 L of it.
A gradient element outside the entries is (Q r_p - r_q P) w / T times a weight e / S <= 1, whose error is at most 2^-21
(see the policy loss), the factor's 2 L (Q r_p + r_q P) <= 2 L (Q + r_q); in them (Q + r_q) p - q with the same error of
p and 2^-22 q of q (exp and product in float32). Together (Q + r_q) (2^-21 + 2 L) + 2^-22 q < 6e-6 max(1, Q), beside 2^-22
for the factors' own rounding and products and half a step of the gradient's type.
"""

import numpy as np
import pytest
import torch

import paper_2608_28726_amd as pr
from oracle import distill as odist
from paper_2608_28726_amd import _abi
from tests.gpu_common import require_gpu
from tests.test_gpu_loss import L_ABS, make_rows, name_of, near, on_gpu, raw_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def teacher_of(logits, T, k, rng, near_student=1.0):
    """The k largest of other logits and their log-probs (float32), in shuffled order."""
    n, V = logits.shape
    u = logits.double().numpy() / T[:, None].astype(np.float64)
    u = u * 1.1 + rng.normal(0, near_student, u.shape)
    lse = np.logaddexp.reduce(u, axis=1)
    k = min(k, V)
    ids = np.argpartition(-u, k - 1, axis=1)[:, :k]
    logq = np.take_along_axis(u, ids, 1) - lse[:, None]
    return ids.astype(np.int32), np.minimum(logq, 0.0).astype(np.float32)


def run(d_logits, ids, logq, T, w, tail, grad=True, scale=1.0, workspace=None):
    c = lambda x: torch.tensor(np.ascontiguousarray(x), device="cuda")  # noqa: E731
    return pr.distill_loss(d_logits, c(ids), c(logq), c(T), c(w), tail=tail, grad=grad, grad_scale=scale,
                           workspace=workspace)


def compare(g, o, logq, dtype, scale=1.0, what=""):
    torch.cuda.synchronize()
    assert np.array_equal(g["flags"].cpu().numpy(), o["flags"]), what
    Q = np.maximum(1.0, np.exp(logq.astype(np.float64)).sum(1))
    near(what + "token_loss", g["token_loss"].cpu().numpy(), o["token_loss"], 2 * L_ABS * Q)
    near(what + "mass", g["mass"].cpu().numpy(), o["mass"], 1e-38, 2 * L_ABS + 2.0 ** -23)
    if np.isfinite(o["loss"]):
        weights = np.abs(o["weight"])
        near(what + "loss", g["loss"].cpu().numpy(), [o["loss"]], (weights * 2 * L_ABS * Q).sum())
    else:
        near(what + "loss", g["loss"].cpu().numpy(), [o["loss"]], 0.0)
    if "grad" in g:
        half = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
        near(what + "grad", g["grad"].float().cpu().numpy(), o["grad"],
             6e-6 * np.abs(o["coef"])[:, None] * Q[:, None] + 1e-38, half * 1.01 + 2.0 ** -22)


def oracle_of(logits, ids, logq, T, w, tail, scale=1.0):
    o = odist.distill_loss(raw_of(logits), name_of(logits.dtype), ids, logq, T, w, tail, scale)
    o["weight"] = w.astype(np.float64)
    return o


SHAPES = [
    # n, V, k, dtype, pad, start
    (1, 2, 1, torch.float32, 0, 0),
    (1, 2, 2, torch.bfloat16, 0, 1),
    (3, 3, 2, torch.bfloat16, 0, 1),
    (5, 7, 7, torch.bfloat16, 0, 0),
    (4, 9, 5, torch.float32, 3, 1),
    (17, 1000, 20, torch.float32, 5, 3),
    (9, 1537, 256, torch.bfloat16, 11, 5),
    (4, 50257, 64, torch.bfloat16, 0, 0),
    (3, 50257, 256, torch.float32, 0, 2),
    (3, 32000, 20, torch.float32, 0, 0),
    (2, 151936, 64, torch.bfloat16, 0, 0),
    (2, 151936, 100, torch.float32, 64, 0),
    (2, 262144, 256, torch.float32, 0, 0),
    (2, 262147, 33, torch.bfloat16, 0, 7),
    (300, 257, 17, torch.float32, 0, 0),
    (1500, 65, 8, torch.bfloat16, 0, 0),
    (40, 30011, 12, torch.bfloat16, 0, 0),
    (70, 20000, 31, torch.float32, 0, 0),
    (300, 40000, 48, torch.bfloat16, 0, 3),
]
# On either side of where rows are held by a workgroup or spread over several.
SHAPES += [(n, V, k, dtype, 0, start)
           for n, k, start in ((300, 33, 0), (300, 256, 1))
           for V, dtype in ((4095, torch.bfloat16), (4096, torch.bfloat16), (2051, torch.float32))] + [
    (8200, 4096, 32, torch.bfloat16, 0, 1), (8200, 2051, 33, torch.float32, 0, 0),
    (12, 32000, 64, torch.float32, 0, 0), (13, 32000, 64, torch.float32, 0, 3), (31, 32000, 65, torch.float32, 0, 1),
    (32, 32000, 65, torch.float32, 0, 0), (25, 40003, 20, torch.float32, 0, 0), (26, 40003, 20, torch.float32, 0, 1),
    (255, 4100, 20, torch.bfloat16, 0, 1), (255, 4090, 256, torch.bfloat16, 0, 1),
]


@pytest.mark.parametrize("tail", ["rest", "drop", "renorm"])
@pytest.mark.parametrize("n,V,k,dtype,pad,start", SHAPES)
def test_against_the_oracle(n, V, k, dtype, pad, start, tail):
    print("case", n, V, k, dtype, pad, start, tail, flush=True)
    buf, logits, _, T, rng = make_rows(n, V, dtype, 17 * n + V, pad, start)
    ids, logq = teacher_of(logits, T, k, rng)
    w = rng.uniform(0.1, 1.0, n).astype(np.float32)
    if n > 1:
        w[rng.random(n) < 0.25] = 0.0
        logq[rng.random(logq.shape) < 0.1] = -np.inf  # entries that are none
        ids[np.isneginf(logq)] = -7
    if n > 4:
        w[3] = -w[3]
        logq[2] = -np.inf
    g = run(on_gpu(buf, logits), ids, logq, T, w, tail, scale=0.5)
    compare(g, oracle_of(logits, ids, logq, T, w, tail, 0.5), logq, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V", [(5, 50257), (3, 151936), (100, 30000), (300, 4001), (270, 40000)])
def test_in_place_strided_and_without_gradient(n, V, dtype):
    """The gradient in the logits' place, in rows apart and at another alignment, and none at all: the same values."""
    buf, logits, _, T, rng = make_rows(n, V, dtype, n + V, 3, 1)
    ids, logq = teacher_of(logits, T, 20, rng)
    w = np.where(rng.random(n) < 0.2, 0.0, 1.0 / n).astype(np.float32)
    o = oracle_of(logits, ids, logq, T, w, "rest")
    first = run(on_gpu(buf, logits), ids, logq, T, w, "rest")
    compare(first, o, logq, dtype)
    d = on_gpu(buf, logits)
    there = run(d, ids, logq, T, w, "rest", grad=d)
    assert there["grad"].data_ptr() == d.data_ptr()
    wide = torch.full((n, V + 5), 7.0, dtype=dtype, device="cuda")
    apart = run(on_gpu(buf, logits), ids, logq, T, w, "rest", grad=wide[:, 2:V + 2])
    none = run(on_gpu(buf, logits), ids, logq, T, w, "rest", grad=False)
    torch.cuda.synchronize()
    assert "grad" not in none
    compare(none, o, logq, dtype)
    assert torch.equal(there["grad"], first["grad"]) and torch.equal(apart["grad"], first["grad"])
    assert (wide[:, :2] == 7).all() and (wide[:, V + 2:] == 7).all()
    for name in ("loss", "token_loss", "mass", "flags"):
        assert torch.equal(there[name], first[name]) and torch.equal(apart[name], first[name])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,V", [(12, 37), (12, 30011), (300, 30011)])
@pytest.mark.parametrize("tail", ["rest", "drop", "renorm"])
def test_special_rows(n, V, dtype, tail):
    """Masked rows full of NaN, bad logits, temperatures and entries, ids twice, impossible tokens, nothing left over."""
    buf, logits, _, T, rng = make_rows(n, V, dtype, 3, 1, 0)
    ids, logq = teacher_of(logits, T, 9, rng)
    w = np.ones(n, np.float32)
    logits[0], w[0], T[0] = float("nan"), 0.0, -1.0
    logits[1, V // 2] = float("nan")
    logits[2, V - 1] = float("inf")
    logits[3] = float("-inf")
    T[4] = 0.0
    ids[5, 2] = ids[5, 7]
    ids[6, 1] = V
    ids[7, 0], logq[7, 0] = -1, np.nan
    logq[8, 4] = np.inf
    keep = logits[9, ids[9].astype(np.int64)].clone()
    logits[9] = float("-inf")
    logits[9, ids[9].astype(np.int64)] = keep  # no other token is left
    logits[10, int(ids[10, 0])] = float("-inf")  # a token of the teacher's that the student cannot say
    ids[11, 3:], logq[11, 3:] = ids[11, 0], -np.inf  # ids of entries that are none may be anything
    g = run(on_gpu(buf, logits), ids, logq, T, w, tail)
    o = oracle_of(logits, ids, logq, T, w, tail)
    assert o["flags"][:12].tolist() == [16, 1, 1, 1, 4, 2, 2, 3, 1, 0, 0, 0] and o["token_loss"][10] == np.inf
    compare(g, o, logq, dtype)


def test_infinite_loss():
    z = torch.zeros(1, 50, device="cuda")
    z[0, 3] = float("-inf")
    g = run(z, np.array([[3, 4]], np.int32), np.log(np.array([[0.5, 0.25]], np.float32)), np.ones(1, np.float32),
            np.ones(1, np.float32), "rest")
    torch.cuda.synchronize()
    assert torch.isinf(g["loss"]).all() and torch.isfinite(g["grad"]).all() and g["grad"][0, 3] == -0.5


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_student_that_is_sure(dtype):
    """The rest's probability is far below 2^-24 and keeps its precision: 60 to 90 nats below the entries."""
    n, V = 4, 5000
    rng = np.random.default_rng(0)
    logits = torch.tensor(rng.normal(0, 1, (n, V))).to(dtype)
    ids = np.stack([rng.permutation(V)[:6] for _ in range(n)]).astype(np.int32)
    for r in range(n):
        logits[r, ids[r].astype(np.int64)] += 70 + 10 * r
    T = np.ones(n, np.float32)
    logq = np.log(rng.dirichlet(np.ones(6), n) * np.array([0.5, 0.9, 0.99, 1 - 1e-6])[:, None]).astype(np.float32)
    w = np.ones(n, np.float32)
    g = run(logits.cuda(), ids, logq, T, w, "rest")
    compare(g, oracle_of(logits, ids, logq, T, w, "rest"), logq, dtype)


def test_strides_of_the_entries():
    """The first entries of a longer list, and lists whose rows lie apart differently."""
    buf, logits, _, T, rng = make_rows(7, 3001, torch.float32, 8)
    ids, logq = teacher_of(logits, T, 40, rng)
    w = np.ones(7, np.float32)
    d, t = logits.cuda(), torch.tensor
    want = run(d, ids[:, :16], logq[:, :16], T, w, "rest")
    a = pr.distill_loss(d, t(ids).cuda()[:, :16], t(logq).cuda()[:, :16], t(T).cuda(), t(w).cuda())
    b = pr.distill_loss(d, t(ids).cuda()[:, :16], t(np.ascontiguousarray(logq[:, :16])).cuda(), t(T).cuda(), t(w).cuda())
    torch.cuda.synchronize()
    for g in (a, b):
        assert torch.equal(g["grad"], want["grad"]) and torch.equal(g["token_loss"], want["token_loss"])


def test_no_entries_no_rows_and_many():
    z = torch.randn(3, 100, device="cuda")
    one = torch.ones(3, device="cuda")
    e, f = torch.empty(3, 0, dtype=torch.int32, device="cuda"), torch.empty(3, 0, device="cuda")
    for tail in ("drop", "renorm", "rest"):
        g = pr.distill_loss(z, e, f, 1.0, one, tail=tail)
        torch.cuda.synchronize()
        assert g["loss"].item() == 0.0 and g["grad"].abs().max().item() < 1e-6 and (g["mass"] == 0).all()
        g = pr.distill_loss(z[:0], e[:0], f[:0], 1.0, one[:0], tail=tail)
        torch.cuda.synchronize()
        assert g["loss"].item() == 0.0 and g["grad"].shape == (0, 100)
    with pytest.raises(ValueError):
        pr.distill_loss(z, torch.zeros(3, 257, dtype=torch.int32, device="cuda"), torch.zeros(3, 257, device="cuda"), 1.0, one)


def test_repeatable_and_captured():
    """The same call gives the same bits; captured calls that share nothing give them on every replay."""
    cases = []
    for n, V, k in ((6, 50257, 64), (300, 30011, 20), (33, 2000, 256)):
        buf, logits, _, T, rng = make_rows(n, V, torch.bfloat16, n)
        ids, logq = teacher_of(logits, T, k, rng)
        w = np.full(n, 1.0 / n, np.float32)
        c = lambda x: torch.tensor(x, device="cuda")  # noqa: E731
        cases.append((logits.cuda(), c(ids), c(logq), c(T), c(w)))
    eager = [pr.distill_loss(*x) for x in cases]
    again = [pr.distill_loss(*x) for x in cases]
    torch.cuda.synchronize()
    for a, b in zip(eager, again):
        assert all(torch.equal(a[k], b[k]) for k in a)
    graphs = []
    for x in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = pr.distill_loss(*x)
        graphs.append((g, out))
    for _ in range(4):
        for (g, out), want in zip(graphs, eager):
            for t in out.values():
                t.fill_(3)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(out[k], want[k]) for k in want)


def test_on_another_stream_with_a_workspace():
    buf, logits, _, T, rng = make_rows(20, 40000, torch.float32, 4)
    ids, logq = teacher_of(logits, T, 30, rng)
    w = np.ones(20, np.float32)
    want = run(logits.cuda(), ids, logq, T, w, "rest")
    need = _abi.lib().pr_distill_loss_workspace(_abi.PR_F32, 20, 40000, 30)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = run(logits.cuda(), ids, logq, T, w, "rest", workspace=ws)
    s.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(got[k], want[k]) for k in want)


def test_long_rows():
    """More vectors than one bit map marks."""
    n, V, k = 2, 600_011, 256
    buf, logits, _, T, rng = make_rows(n, V, torch.float32, 12, 0, 3)
    ids, logq = teacher_of(logits, T, k, rng)
    w = np.ones(n, np.float32)
    g = run(on_gpu(buf, logits), ids, logq, T, w, "rest")
    compare(g, oracle_of(logits, ids, logq, T, w, "rest"), logq, torch.float32)


@pytest.mark.parametrize("n,V", [(3, 50257), (70, 20000), (300, 1000), (20, 307300)])
def test_a_student_that_agrees(n, V):
    """One entry of probability near 1 that the student gives nearly the same: p - q keeps the precision of 1 - p.

    The entry's exponential and the sum over the entries are the same number. The others' sum o beside it is off by: the
    exponent's scale, 2^-24 of at most 30 nats, 1.8e-6; the rounded difference of the two parts' exponents (below 64 in
    base 2), 2^-19 ln 2 = 1.3e-6; exponentials and sums 2^-21. Together below 4e-6, so p = 1 / (1 + o) is off by
    4e-6 p (1 - p); what follows is in 64 bits.
    """
    rng = np.random.default_rng(V)
    logits = torch.tensor(rng.normal(0, 1, (n, V)), dtype=torch.float32)
    y = rng.integers(0, V, n)
    logits[torch.arange(n), torch.tensor(y)] = torch.tensor(rng.uniform(18, 24, n), dtype=torch.float32)
    z = logits.double().numpy()
    p = np.exp(z[np.arange(n), y] - np.log(np.exp(z - 24).sum(1)) - 24)
    logq = np.log(p * (1 + 1e-4 * rng.normal(0, 1, n)).clip(max=1.0)).astype(np.float32)[:, None]
    ids, T, w = y.astype(np.int32)[:, None], np.ones(n, np.float32), np.ones(n, np.float32)
    g = run(logits.cuda(), ids, logq, T, w, "drop")["grad"][torch.arange(n), torch.tensor(y)].double().cpu().numpy()
    q = np.exp(logq[:, 0].astype(np.float64))
    exact = q * p - q
    assert (np.abs(g - exact) <= 4e-6 * p * (1 - p) + 2.0 ** -24 * np.abs(exact) + 1e-14).all(), (g, exact)
