"""The policy and preference losses and their gradients: HIP path vs the fp64
oracle.

Tolerances. A row's sum of exps: its terms 2^x are off by at most
|x| 2^-23 ln 2 (the argument's and the scale's rounding) + 2^-23 (the exp), and
sum p |x| is at most the row's entropy in bits, below 18; with the sums' own
roundings l is within 2e-6 of the exact one, and 2^-24 |l| for its float32.
What follows from l (ratio, KL, coefficients) carries that error on. A gradient
element coef (delta - p) has p's relative error, at most (|x| + 2) 2^-22, and
p |x| is below 0.54: an absolute error of 2^-21 |coef|, besides the
coefficient's own and the rounding to the gradient's type.
"""

import math

import numpy as np
import pytest
import torch

import paper_2608_28726_amd as pr
from oracle import loss as oloss
from paper_2608_28726_amd import _abi
from paper_2608_28726_amd import workloads as wl
from tests.gpu_common import require_gpu

pytestmark = pytest.mark.gpu

L_ABS = 2e-6


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def make_rows(n, V, dtype, seed, pad=0, start=0):
    """n rows of V logits in a buffer of row stride V + pad whose first row starts `start` elements in; ids drawn by
    Gumbel races; temperatures; log-probs of the ids (float64)."""
    rng = np.random.default_rng(seed)
    z = rng.normal(0, 1, (n, V)) * rng.uniform(0.5, 4.0, (n, 1))
    z[np.arange(n), rng.integers(0, V, n)] += rng.uniform(0, 15, n)
    buf = torch.zeros(n * (V + pad) + start + 8, dtype=dtype)
    logits = buf[start:start + n * (V + pad)].view(n, V + pad)[:, :V]
    logits.copy_(torch.tensor(z))
    T = rng.uniform(0.5, 1.3, n).astype(np.float32)
    u = logits.double().numpy() / T[:, None].astype(np.float64)
    ids = np.argmax(u + rng.gumbel(size=u.shape), axis=1).astype(np.int32)
    return buf, logits, ids, T, rng


def raw_of(logits):
    return wl.to_host_raw(logits)


def name_of(dtype):
    return "bf16" if dtype == torch.bfloat16 else "f32"


def on_gpu(buf, logits):
    """The same rows, at the same place of a device buffer."""
    d = buf.cuda()
    return d.as_strided(logits.size(), logits.stride(), logits.storage_offset())


def near(name, got, want, atol, rtol=2.0 ** -23):
    got = np.asarray(got, dtype=np.float64)
    want = np.asarray(want, dtype=np.float64)
    assert got.shape == want.shape, name
    bad = ~((np.isnan(got) & np.isnan(want)) | (got == want))
    with np.errstate(invalid="ignore"):
        bad &= ~(np.abs(got - want) <= atol + rtol * np.abs(want))
    if bad.any():
        i = tuple(np.argwhere(bad)[0])
        raise AssertionError(f"{name}: {bad.sum()} of {bad.size} off, first at {i}: got {got[i]}, want {want[i]}")


def near_gradient(got, o, T, dtype, coef_rel, scale=1.0):
    """Element tolerance of the module docstring; coef_rel: the coefficients' relative error."""
    g = got.float().cpu().numpy()
    coef = np.nan_to_num(np.abs(o["dl"] / T.astype(np.float64)) * scale)[:, None]
    half_ulp = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24  # 8 and 24 significant bits
    want = o["grad"]
    near("grad", g, want, coef * (2.0 ** -21 + coef_rel) + 1e-38, half_ulp * 1.01 + coef_rel)


POLICY_SHAPES = [
    # n, V, dtype, pad, start: one row, odd vocabularies, rows that start anywhere, rows apart, several sizes of a row
    (1, 2, torch.float32, 0, 0),
    (3, 3, torch.bfloat16, 0, 1),
    (5, 7, torch.bfloat16, 0, 0),
    (2, 1, torch.float32, 3, 1),
    (17, 1000, torch.float32, 5, 3),
    (9, 1537, torch.bfloat16, 11, 5),
    (4, 50257, torch.bfloat16, 0, 0),
    (3, 50257, torch.float32, 0, 2),
    (3, 32000, torch.float32, 0, 0),
    (2, 151936, torch.bfloat16, 0, 0),
    (2, 151936, torch.float32, 64, 0),
    (2, 262144, torch.float32, 0, 0),
    (2, 262147, torch.bfloat16, 0, 7),
    (300, 257, torch.float32, 0, 0),
    (1500, 65, torch.bfloat16, 0, 0),
]
POLICY_SHAPES = [s for s in POLICY_SHAPES if s[1] >= 2]


def policy_inputs(n, V, dtype, pad, start, seed, masked=0.25):
    buf, logits, ids, T, rng = make_rows(n, V, dtype, seed, pad, start)
    u = logits.double().numpy() / T[:, None].astype(np.float64)
    l = u[np.arange(n), ids] - np.logaddexp.reduce(u, axis=1)
    delta = rng.normal(0, 0.3, n)
    delta += np.where(np.abs(delta - math.log(0.8)) < 1e-3, 3e-3, 0.0) + np.where(np.abs(delta - math.log(1.3)) < 1e-3,
                                                                                 3e-3, 0.0)
    old, ref = (l - delta).astype(np.float32), (l + rng.normal(0, 0.4, n)).astype(np.float32)
    A = rng.normal(0.2, 1.0, n).astype(np.float32)
    w = rng.uniform(0.1, 1.0, n).astype(np.float32)
    if n > 1:
        w[rng.random(n) < masked] = 0.0
    return buf, logits, ids, T, w, A, old, ref


@pytest.mark.parametrize("use_ref", [True, False])
@pytest.mark.parametrize("n,V,dtype,pad,start", POLICY_SHAPES)
def test_policy(n, V, dtype, pad, start, use_ref):
    print(f"case policy n={n} V={V} {dtype} pad={pad} start={start} ref={use_ref}", flush=True)
    buf, logits, ids, T, w, A, old, ref = policy_inputs(n, V, dtype, pad, start, 100 + n + V)
    kl = 0.07 if use_ref else 0.0
    ref = ref if use_ref else None
    o = oloss.policy_loss(raw_of(logits), name_of(dtype), ids, T, w, A, old, ref, 0.2, 0.3, kl, 2.5)
    d = on_gpu(buf, logits)
    cu = lambda x: None if x is None else torch.tensor(x, device="cuda")  # noqa: E731
    got = pr.policy_loss(d, cu(ids), cu(T), cu(w), cu(A), cu(old), cu(ref), clip_low=0.2, clip_high=0.3, kl_coef=kl,
                         grad_scale=2.5)
    torch.cuda.synchronize()
    near("logprob", got["logprob"].cpu(), o["logprob"], L_ABS)
    near("ratio", got["ratio"].cpu(), o["ratio"], 0.0, 2 * L_ABS)
    near("kl", got["kl"].cpu(), o["kl"], L_ABS * (1 + 2 * np.abs(o["kl"])), 2.0 ** -23)
    assert got["flags"].cpu().numpy().tolist() == o["flags"].tolist()
    reach = float(np.sum(np.abs(w) * (np.abs(A) * o["ratio"] + kl * np.exp(np.abs(o["kl"])))))
    near("loss", got["loss"].cpu(), [o["loss"]], 2 * L_ABS * reach)
    near_gradient(got["grad"], o, T, dtype, 2 * L_ABS * (1 + 10 * kl), 2.5)
    # without the gradient the rest is the same
    less = pr.policy_loss(d, cu(ids), cu(T), cu(w), cu(A), cu(old), cu(ref), clip_low=0.2, clip_high=0.3, kl_coef=kl,
                          grad=False)
    assert "grad" not in less
    near("loss alone", less["loss"].cpu(), [o["loss"]], 2 * L_ABS * reach)
    near("logprob alone", less["logprob"].cpu(), o["logprob"], L_ABS)
    # the same inputs give the same bits, also in the logits' place
    again = pr.policy_loss(d, cu(ids), cu(T), cu(w), cu(A), cu(old), cu(ref), clip_low=0.2, clip_high=0.3, kl_coef=kl,
                           grad_scale=2.5, grad=d)
    assert again["grad"] is d
    for k in ("loss", "logprob", "ratio", "kl", "grad"):
        assert torch.equal(again[k], got[k]), k
    # and the elements between rows are left alone
    if pad and n > 1:
        assert bool((d.as_strided((n - 1, pad), (V + pad, 1), d.storage_offset() + V) == 0).all())


@pytest.mark.parametrize("n,V,dtype,pad", [(70001, 9, torch.float32, 0), (66000, 40, torch.bfloat16, 3),
                                           (2500, 3001, torch.bfloat16, 0), (1100, 8000, torch.float32, 1),
                                           (600, 32000, torch.float32, 0), (1300, 50257, torch.bfloat16, 0),
                                           (300, 70001, torch.float32, 0), (600, 151936, torch.bfloat16, 0),
                                           (1030, 170000, torch.bfloat16, 0)])
def test_policy_many_rows(n, V, dtype, pad):
    """Batches that take every workgroup several rows, in each size of a row, listed or not, against plain float64
    operations on the device."""
    print(f"case policy many n={n} V={V} {dtype}", flush=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    logits = torch.empty(n, V + pad, device="cuda").normal_(generator=g).mul_(3.0).to(dtype)[:, :V]
    ids = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    T = torch.rand(n, generator=g, device="cuda") + 0.5
    w = torch.rand(n, generator=g, device="cuda") + 0.1
    w[torch.rand(n, generator=g, device="cuda") < 0.3] = 0.0
    if n > 20:
        w[5:17] = 0.0
    on = w != 0
    logits[~on] = math.nan
    A = torch.empty(n, device="cuda").normal_(generator=g)
    l = torch.zeros(n, dtype=torch.float64, device="cuda")
    step = max(1, 200_000_000 // V)
    for a in range(0, n, step):
        u = logits[a:a + step].double() / T[a:a + step, None].double()
        l[a:a + step] = torch.log_softmax(u, 1).gather(1, ids[a:a + step, None].long())[:, 0]
    delta = torch.empty(n, device="cuda").normal_(generator=g).mul_(0.3)
    delta = torch.where((delta.exp() - 0.8).abs() < 2e-3, delta + 0.01, delta)
    delta = torch.where((delta.exp() - 1.2).abs() < 2e-3, delta + 0.01, delta)
    old = torch.where(on, (l - delta).float(), 0.0)
    got = pr.policy_loss(logits, ids, T, w, A, old, grad_scale=0.5)
    torch.cuda.synchronize()
    ratio = torch.exp(l - old.double())
    free, held = ratio * A, ratio.clamp(0.8, 1.2) * A
    clipped = on & (free > held)
    terms = torch.where(on, -w.double() * torch.minimum(free, held), 0.0)
    assert torch.equal(got["flags"], torch.where(on, torch.where(clipped, pr.FLAG_CLIPPED, 0), pr.FLAG_MASKED).int())
    near("logprob", got["logprob"].cpu(), torch.where(on, l, 0.0).cpu(), L_ABS)
    near("loss", got["loss"].cpu(), [float(terms.sum())], 2 * L_ABS * float(terms.abs().sum()))
    coef = torch.where(on, 0.5 * w.double() * torch.where(clipped, 0.0, -free) / T.double(), 0.0)
    half_ulp = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    for a in range(0, n, step):
        rows = slice(a, a + step)
        u = logits[rows].double() / T[rows, None].double()
        want = -torch.softmax(u, 1)
        want.scatter_add_(1, ids[rows, None].long(), torch.ones_like(want[:, :1]))
        want = torch.where(on[rows, None], want * coef[rows, None], 0.0)
        off = (got["grad"][rows].double() - want).abs()
        allowed = coef[rows, None].abs() * (2.0 ** -21 + 2 * L_ABS) + (half_ulp * 1.01 + 2 * L_ABS) * want.abs() + 1e-38
        bad = ~(off <= allowed)
        assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:3].tolist())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [65, 4096, 50257])
def test_policy_gradient_elsewhere(V, dtype):
    """A gradient whose rows sit otherwise than the logits' (stride and start)."""
    n = 6
    buf, logits, ids, T, w, A, old, ref = policy_inputs(n, V, dtype, 0, 0, 5)
    o = oloss.policy_loss(raw_of(logits), name_of(dtype), ids, T, w, A, old, ref, kl_coef=0.05)
    d = on_gpu(buf, logits)
    flat = torch.full((n * (V + 3) + 9,), 7.0, dtype=dtype, device="cuda")
    g = flat[1:1 + n * (V + 3)].view(n, V + 3)[:, 2:V + 2]
    cu = lambda x: torch.tensor(x, device="cuda")  # noqa: E731
    pr.policy_loss(d, cu(ids), cu(T), cu(w), cu(A), cu(old), cu(ref), kl_coef=0.05, grad=g)
    near_gradient(g, o, T, dtype, 3 * L_ABS)
    rest = flat.clone()
    rest[1:1 + n * (V + 3)].view(n, V + 3)[:, 2:V + 2] = 7.0
    assert bool((rest == 7.0).all())


def special_rows(V, dtype):
    """Rows at the limits: (logits, id, temperature, what is flagged)."""
    inf, low = math.inf, torch.finfo(dtype).min
    base = np.random.default_rng(3).normal(0, 2, V)

    def row(**at):
        r = base.copy()
        for k, v in at.items():
            r[int(k[1:]) % V] = v
        return r

    masked = np.full(V, -inf)
    masked[V - 1] = 1.0
    lows = np.full(V, low)
    lows[[0, V // 2]] = [1.0, 2.0]
    return [
        (row(), 0, 1.0, 0),
        (row(i5=-inf, i1=-inf), 0, 1.0, 0),                  # tokens that the decoder forbids
        (masked, V - 1, 0.7, 0),                             # one token left
        (lows, 0, 1.0, 0),                                   # masks of the type's lowest value
        (np.full(V, 0.25), V // 2, 0.5, 0),                  # uniform
        (row(i3=40.0), 3, 1.0, 0),                           # all but certain
        (row(i3=300.0), 4 % V, 1.0, 0),                      # all but impossible
        (base + 3e4, 1, 1.0, 0),                             # far from zero
        (row(i2=math.nan), 0, 1.0, oloss.FLAG_NONFINITE),
        (row(i2=inf), 0, 1.0, oloss.FLAG_NONFINITE),
        (np.full(V, -inf), 0, 1.0, oloss.FLAG_NONFINITE),
        (row(), V, 1.0, oloss.FLAG_BAD_ID),
        (row(), -1, 1.0, oloss.FLAG_BAD_ID),
        (row(), 1, 0.0, oloss.FLAG_BAD_TP),
        (row(), 1, math.nan, oloss.FLAG_BAD_TP),
    ]


@pytest.mark.parametrize("V", [8, 700, 33000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_policy_special_rows(V, dtype):
    """Each row at the limits, counted and not: what does not count is not read, what is bad says so."""
    rows = special_rows(V, dtype)
    n = len(rows)
    logits = torch.tensor(np.stack([r[0] for r in rows])).to(dtype)
    ids = np.array([r[1] for r in rows], np.int32)
    T = np.array([r[2] for r in rows], np.float32)
    A = np.linspace(-1, 1.5, n).astype(np.float32)
    cu = lambda x: torch.tensor(x, device="cuda")  # noqa: E731
    for count in (range(8), range(n), range(8, n)):
        w = np.zeros(n, np.float32)
        w[list(count)] = 0.5
        old = np.full(n, -3.0, np.float32)
        fine = oloss.policy_loss(raw_of(logits), name_of(dtype), ids, T, np.where(np.arange(n) < 8, 1.0, 0.0), A, old)
        old[:8] = fine["logprob"][:8].clip(min=-80.0) - 0.1
        o = oloss.policy_loss(raw_of(logits), name_of(dtype), ids, T, w, A, old)
        got = pr.policy_loss(logits.cuda(), cu(ids), cu(T), cu(w), cu(A), cu(old))
        torch.cuda.synchronize()
        assert got["flags"].cpu().tolist() == o["flags"].tolist()
        # far from zero the float32 row reference moves l by its residual's rounding
        near("logprob", got["logprob"].cpu(), o["logprob"], 4 * L_ABS)
        ok = np.arange(n) < 8
        near_gradient(got["grad"][:8], {"dl": o["dl"][ok], "grad": o["grad"][ok]}, T[ok], dtype, 2e-5)
        g = got["grad"].float().cpu().numpy()
        for r in range(8, n):
            assert np.isnan(g[r]).all() if w[r] else (g[r] == 0).all()
        assert math.isnan(float(got["loss"])) == (max(count) >= 8)


@pytest.mark.parametrize("V,dtype", [(30000, torch.float32), (60000, torch.bfloat16), (40000, torch.float32),
                                     (80000, torch.bfloat16)])
def test_policy_special_rows_held(V, dtype):
    """The special rows among many rows, of the sizes that a workgroup holds: all count, then only the good ones."""
    base = special_rows(V, dtype)
    k, times = len(base), 128 // len(base) + 1
    n = k * times
    logits = torch.tensor(np.stack([r[0] for r in base])).to(dtype)
    ids = np.array([r[1] for r in base], np.int32)
    T = np.array([r[2] for r in base], np.float32)
    A = np.linspace(-1, 1.5, k).astype(np.float32)
    good = np.arange(k) < 8
    fine = oloss.policy_loss(raw_of(logits), name_of(dtype), ids, T, np.where(good, 1.0, 0.0), A, np.full(k, -3.0, np.float32))
    old = np.full(k, -3.0, np.float32)
    old[:8] = fine["logprob"][:8].clip(min=-80.0) - 0.1
    cu = lambda x: torch.tensor(np.tile(x, times), device="cuda")  # noqa: E731
    for w in (np.full(k, 0.5, np.float32), np.where(good, 0.5, 0.0).astype(np.float32)):
        o = oloss.policy_loss(raw_of(logits), name_of(dtype), ids, T, w, A, old)
        got = pr.policy_loss(logits.cuda().repeat(times, 1), cu(ids), cu(T), cu(w), cu(A), cu(old))
        torch.cuda.synchronize()
        assert got["flags"].cpu().tolist() == o["flags"].tolist() * times
        near("logprob", got["logprob"].cpu(), np.tile(o["logprob"], times), 4 * L_ABS)
        g = got["grad"].view(times, k, V)
        # the loss is a mean over the rows: `times` as many rows, if the weights are normed by their count
        for t in range(times):
            near_gradient(g[t, :8], {"dl": o["dl"][good], "grad": o["grad"][good]}, T[good], dtype, 2e-5)
            bad = g[t, 8:].float().cpu().numpy()
            assert np.isnan(bad).all() if w[8] else (bad == 0).all()
        assert math.isnan(float(got["loss"])) == bool(w[8])


@pytest.mark.parametrize("n", [3, 50, 700])
@pytest.mark.parametrize("V", [1000, 70000])
def test_policy_clipped_rows_with_forbidden_tokens(n, V):
    """Rows whose gradient is 0 because the ratio is clipped, with logits of -inf among them: 0 everywhere, in each way
    that rows are dealt out; rows beside them as the oracle has them."""
    if n * V > 4_000_000:
        n = 40
    rng = np.random.default_rng(n)
    z = rng.normal(0, 2, (n, V)).astype(np.float32)
    z[:, V // 3:V // 2] = -np.inf
    ids = rng.integers(0, V // 3, n).astype(np.int32)
    u = z.astype(np.float64)
    l = u[np.arange(n), ids] - np.logaddexp.reduce(u, axis=1)
    up = np.arange(n) % 2 == 0
    old = np.where(up, l - 1.0, l).astype(np.float32)  # every other ratio is e, past the clip
    A, w, T = np.ones(n, np.float32), np.ones(n, np.float32), np.ones(n, np.float32)
    cu = lambda x: torch.tensor(x, device="cuda")  # noqa: E731
    got = pr.policy_loss(cu(z), cu(ids), cu(T), cu(w), cu(A), cu(old))
    torch.cuda.synchronize()
    g = got["grad"].cpu().numpy()
    assert np.isfinite(g).all() and (g[up] == 0).all()
    assert ((got["flags"].cpu().numpy() == pr.FLAG_CLIPPED) == up).all()
    if not up.all():
        o = oloss.policy_loss(z[1:2], "f32", ids[1:2], T[1:2], w[1:2], A[1:2], old[1:2])
        near_gradient(got["grad"][1:2], o, T[1:2], torch.float32, 2 * L_ABS)


def test_policy_probability_zero():
    """A token of probability 0: ratio 0; with a KL term the loss is infinite, as the formula has it."""
    logits = torch.zeros(1, 16, device="cuda")
    logits[0, 3] = -math.inf
    one = torch.ones(1, device="cuda")
    ids = torch.tensor([3], dtype=torch.int32, device="cuda")
    got = pr.policy_loss(logits, ids, one, one, one, -one)
    assert float(got["logprob"]) == -math.inf and float(got["ratio"]) == 0.0 and float(got["loss"]) == 0.0
    assert bool((got["grad"] == 0).all()) and int(got["flags"]) == 0
    got = pr.policy_loss(logits, ids, one, one, one, -one, -one, kl_coef=0.1)
    assert float(got["kl"]) == math.inf and float(got["loss"]) == math.inf


def test_policy_kl_beside_a_loss_without_it():
    """kl_coef = 0 with a reference: the KL is an output alone, infinite at a token of probability 0, and loss and
    gradient do without it."""
    logits = torch.randn(3, 300, device="cuda")
    logits[1, 7] = -math.inf
    one = torch.ones(3, device="cuda")
    ids = torch.full((3,), 7, dtype=torch.int32, device="cuda")
    plain = pr.policy_loss(logits, ids, one, one, one, -one)
    got = pr.policy_loss(logits, ids, one, one, one, -one, -one)
    assert float(got["kl"][1]) == math.inf and math.isfinite(float(got["loss"]))
    for k in ("loss", "grad", "ratio", "flags"):
        assert torch.equal(got[k], plain[k]), k
    assert bool((got["grad"][1] == 0).all())


@pytest.mark.parametrize("V", [64, 40000])
def test_policy_ratio_beyond_float32(V):
    """A ratio of e^100: clipped at a positive advantage, worth nothing at an advantage of 0, and finite again under a
    weight that brings it back into range."""
    n = 200
    logits = torch.zeros(n, V, device="cuda")
    l = -math.log(V)
    A = torch.tensor([1.0, 0.0, -1.0, 0.0], device="cuda").repeat(n // 4)
    w = torch.tensor([1.0, 1.0, 1e-30, 0.5], device="cuda").repeat(n // 4)
    old = torch.full((n,), l - 100.0, device="cuda")
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")
    got = pr.policy_loss(logits, ids, 1.0, w, A, old)
    x = l - float(old[0])  # with old's rounding
    push = float(w[2]) * math.exp(x)
    assert bool((got["ratio"] == math.inf).all())
    # the exponent's argument is off by L_ABS, the exponential by two roundings of float32
    near("loss", got["loss"].cpu(), [n // 4 * (push - 1.2)], 0.0, L_ABS + 2.0 ** -21)
    want = torch.zeros(n, V, dtype=torch.float64)
    want[2::4] = -push / V
    want[2::4, 0] = push * (1 - 1 / V)
    near("grad", got["grad"].cpu(), want, push * 2.0 ** -21, L_ABS + 2.0 ** -21)


def test_policy_all_masked_and_empty():
    logits = torch.full((5, 300), math.nan, device="cuda")
    z = torch.zeros(5, device="cuda")
    ids = torch.full((5,), -7, dtype=torch.int32, device="cuda")
    got = pr.policy_loss(logits, ids, z, z, z, z)
    assert float(got["loss"]) == 0.0 and bool((got["grad"] == 0).all()) and bool((got["flags"] == pr.FLAG_MASKED).all())
    got = pr.policy_loss(logits[:0], ids[:0], z[:0], z[:0], z[:0], z[:0])
    assert float(got["loss"]) == 0.0 and got["grad"].shape == (0, 300)


PREFERENCE_SHAPES = [
    # lengths of the requests, V, dtype, pad, start
    ([1, 1], 2, torch.float32, 0, 0),
    ([3, 2], 7, torch.bfloat16, 0, 1),
    ([0, 4, 2, 0, 1, 5], 1000, torch.float32, 3, 1),
    ([0, 0], 64, torch.float32, 0, 0),
    ([2, 3], 50257, torch.bfloat16, 0, 0),
    ([1, 2], 151936, torch.bfloat16, 0, 0),
    ([1, 1], 151936, torch.float32, 0, 0),
    ([1, 1], 262144, torch.float32, 0, 0),
    ([130, 70, 400, 5], 129, torch.float32, 0, 0),
    ([600, 700], 65, torch.bfloat16, 0, 0),
]


@pytest.mark.parametrize("options", [dict(), dict(beta=2.0, margin=0.5, ref=False), dict(label_smoothing=0.2)])
@pytest.mark.parametrize("lengths,V,dtype,pad,start", PREFERENCE_SHAPES)
def test_preference(lengths, V, dtype, pad, start, options):
    print(f"case preference {lengths} V={V} {dtype} pad={pad} start={start} {options}", flush=True)
    options = dict(options)
    use_ref = options.pop("ref", True)
    n = sum(lengths)
    buf, logits, ids, T, rng = make_rows(n, V, dtype, 11 + V, pad, start)
    off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    w = (rng.random(n) > 0.2).astype(np.float32) * rng.uniform(0.5, 1.0, n).astype(np.float32)
    u = logits.double().numpy() / T[:, None].astype(np.float64) if n else np.zeros((0, V))
    l = u[np.arange(n), ids] - np.logaddexp.reduce(u, axis=1) if n else np.zeros(0)
    ref = (l + rng.normal(0, 0.3, n)).astype(np.float32) if use_ref else None
    if not use_ref:
        w /= max(lengths) + 1
    o = oloss.preference_loss(raw_of(logits) if n else np.zeros((0, V), np.float32), name_of(dtype), ids, T, w, off,
                              ref, grad_scale=3.0, **options)
    d = on_gpu(buf, logits)
    cu = lambda x: None if x is None else torch.tensor(x, device="cuda")  # noqa: E731
    call = lambda **k: pr.preference_loss(d, cu(ids), cu(T), cu(w), cu(off), cu(ref), **options, **k)  # noqa: E731
    got = call(grad_scale=3.0)
    torch.cuda.synchronize()
    assert got["flags"].cpu().numpy().tolist() == o["flags"].tolist()
    near("logprob", got["logprob"].cpu(), o["logprob"], L_ABS)
    q_abs = L_ABS * max([float(w[off[i]:off[i + 1]].sum()) for i in range(len(lengths))] + [0.0])
    h_abs = 2 * options.get("beta", 0.1) * q_abs
    near("seq_logratio", got["seq_logratio"].cpu(), o["seq_logratio"], q_abs)
    near("pair_logit", got["pair_logit"].cpu(), o["pair_logit"], h_abs)
    near("pair_loss", got["pair_loss"].cpu(), o["pair_loss"], h_abs)
    near("loss", got["loss"].cpu(), [o["loss"]], h_abs)
    # sigma's relative slope is at most 1; with smoothing the two parts may cancel, by at most 1 / |dh|
    dh = np.abs(np.nan_to_num(o["dl"][o["dl"] != 0])).min(initial=1.0)
    coef_rel = h_abs * (1.0 if not options.get("label_smoothing") else max(1.0, 0.1 / dh))
    near_gradient(got["grad"], o, T, dtype, coef_rel + 2.0 ** -23, 3.0)
    less = call(grad=False)
    assert "grad" not in less and torch.equal(less["loss"], got["loss"])
    again = call(grad_scale=3.0, grad=d)
    for k in ("loss", "pair_logit", "seq_logratio", "logprob", "grad"):
        assert torch.equal(again[k], got[k]), k


@pytest.mark.parametrize("n_pairs,most,V,dtype", [(5000, 2, 5, torch.float32), (300, 12, 3001, torch.bfloat16),
                                                  (40, 60, 50257, torch.float32), (2, 900, 200, torch.float32)])
def test_preference_many_pairs(n_pairs, most, V, dtype):
    """Batches of many pairs or long requests (empty ones among them), against plain float64 operations on the device."""
    rng = np.random.default_rng(n_pairs)
    lengths = rng.integers(0, most + 1, 2 * n_pairs)
    off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    n = int(off[-1])
    print(f"case preference many pairs={n_pairs} rows={n} V={V} {dtype}", flush=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    logits = torch.empty(n, V, device="cuda").normal_(generator=g).mul_(3.0).to(dtype)
    ids = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    T = torch.rand(n, generator=g, device="cuda") + 0.5
    w = torch.rand(n, generator=g, device="cuda") + 0.1
    w[torch.rand(n, generator=g, device="cuda") < 0.2] = 0.0
    u = logits.double() / T[:, None].double()
    p = torch.softmax(u, 1)
    l = torch.log_softmax(u, 1).gather(1, ids[:, None].long())[:, 0]
    ref = (l + torch.empty(n, device="cuda").normal_(generator=g) * 0.3).float()
    req = torch.from_numpy(np.repeat(np.arange(2 * n_pairs), lengths)).cuda()
    q = torch.zeros(2 * n_pairs, dtype=torch.float64, device="cuda").index_add_(0, req, w.double() * (l - ref.double()))
    h = 0.3 * (q[0::2] - q[1::2])
    got = pr.preference_loss(logits, ids, T, w, torch.from_numpy(off).cuda(), ref, beta=0.3, grad_scale=n_pairs)
    torch.cuda.synchronize()
    q_abs = L_ABS * most * 1.1
    near("seq_logratio", got["seq_logratio"].cpu(), q.cpu(), q_abs)
    near("pair_logit", got["pair_logit"].cpu(), h.cpu(), 0.6 * q_abs)
    want = torch.nn.functional.softplus(-h)
    near("pair_loss", got["pair_loss"].cpu(), want.cpu(), 0.6 * q_abs)
    near("loss", got["loss"].cpu(), [float(want.mean())], 0.6 * q_abs)
    dq = torch.stack([-torch.sigmoid(-h), torch.sigmoid(-h)], 1).reshape(-1) * 0.3
    coef = (dq[req] * w.double() / T.double())[:, None]
    want = -coef * p
    want.scatter_add_(1, ids[:, None].long(), coef)
    half_ulp = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    rel = 0.6 * q_abs + 2.0 ** -22
    bad = ~((got["grad"].double() - want).abs()
            <= coef.abs() * (2.0 ** -21 + rel) + (half_ulp * 1.01 + rel) * want.abs() + 1e-38)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:3].tolist())
    alone = pr.preference_loss(logits, ids, T, w, torch.from_numpy(off).cuda(), ref, beta=0.3, grad=False)
    assert abs(float(alone["loss"]) - float(got["loss"])) <= 2.0 ** -23 * abs(float(got["loss"]))


def test_preference_bad_and_masked_rows():
    """A bad row spoils its pair and the loss, not the other pair; the same row does nothing when it does not count."""
    V = 515
    buf, logits, ids, T, rng = make_rows(8, V, torch.float32, 2)
    logits[1, 7] = math.nan
    off = np.array([0, 2, 4, 6, 8], np.int32)
    cu = lambda x: torch.tensor(x, device="cuda")  # noqa: E731
    for weight in (1.0, 0.0):
        w = np.ones(8, np.float32)
        w[1] = weight
        o = oloss.preference_loss(raw_of(logits), "f32", ids, T, w, off)
        got = pr.preference_loss(logits.cuda(), cu(ids), cu(T), cu(w), cu(off))
        torch.cuda.synchronize()
        near("loss", got["loss"].cpu(), [o["loss"]], 1e-6)
        near("pair_loss", got["pair_loss"].cpu(), o["pair_loss"], 1e-6)
        near_gradient(got["grad"], o, T, torch.float32, 1e-5)
        g = got["grad"].cpu().numpy()
        assert np.isnan(g[:4]).all() if weight else np.isfinite(g).all()
        assert np.isfinite(g[4:]).all()


def test_preference_saturated():
    """Pairs far apart either way: the loss is the distance or 0, its slope beta or 0, never NaN."""
    z = np.zeros((4, 4), np.float32)
    logits = torch.tensor(z, device="cuda")
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    one = torch.ones(4, device="cuda")
    ref = torch.tensor([-5e4, 0.0, 0.0, -5e4], device="cuda")
    off = torch.arange(5, dtype=torch.int32, device="cuda")
    got = pr.preference_loss(logits, ids, 1.0, one, off, ref, beta=1.0)
    want = oloss.preference_loss(z, "f32", [0] * 4, [1.0] * 4, [1.0] * 4, [0, 1, 2, 3, 4], ref.cpu().numpy(), beta=1.0)
    assert got["pair_loss"].tolist() == [0.0, 5e4] and bool((got["grad"][:2] == 0).all())
    near("grad", got["grad"].cpu(), want["grad"], 1e-6)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_differences(dtype):
    """The gradient against central differences of the kernels' own loss: per-row values are float32, so the step is
    wide and the tolerance takes its curvature, at most coef step^2 / 6 over the step, and the loss's rounding."""
    n, V = 6, 40
    buf, logits, ids, T, w, A, old, ref = policy_inputs(n, V, torch.float32, 0, 0, 77, masked=0.0)
    cu = lambda x: torch.tensor(x, device="cuda")  # noqa: E731
    step = 2.0 ** -5
    z = (logits.float() / step).round() * step  # exact in both types when moved by a step
    z = z.clamp(-7, 7).to(dtype).cuda()
    args = (cu(ids), 1.0, cu(w), cu(A), cu(old), cu(ref))
    # no clipping, so that the loss is smooth
    opts = dict(clip_low=1.0, clip_high=math.inf, kl_coef=0.1)
    base = pr.policy_loss(z.float(), *args, **opts)
    off = torch.tensor([0, 2, 3, 5, 6], dtype=torch.int32, device="cuda")
    pref = lambda x, g: pr.preference_loss(x, args[0], 1.0, args[2], off, args[5], beta=0.7, grad=g)  # noqa: E731
    basep = pref(z.float(), True)
    scale = float((base["ratio"] * args[3].abs() * args[2]).max()) + 0.1 * math.exp(2.0)
    for r, v in ((0, 1), (2, int(ids[2])), (4, 39), (5, int(ids[5]))):
        up, down = z.float().clone(), z.float().clone()
        up[r, v] += step
        down[r, v] -= step
        num = (float(pr.policy_loss(up, *args, grad=False, **opts)["loss"])
               - float(pr.policy_loss(down, *args, grad=False, **opts)["loss"])) / (2 * step)
        assert abs(num - float(base["grad"][r, v])) < scale * step * step + 1e-6 / step * max(1.0, abs(float(base["loss"])))
        num = (float(pref(up, False)["loss"]) - float(pref(down, False)["loss"])) / (2 * step)
        assert abs(num - float(basep["grad"][r, v])) < step * step + 1e-6 / step


def test_more_rows_than_a_launch():
    """More rows, and more pairs, than workgroups whose threads are counted in 32 bits: several launches take them. Two
    tokens a row, whose log-probs are log sigmoids."""
    n_pairs = (1 << 24) + 3
    n = 2 * n_pairs
    print(f"case more rows than a launch n={n}", flush=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    logits = torch.empty(n, 2, device="cuda").normal_(generator=g)
    ids = torch.randint(0, 2, (n,), generator=g, device="cuda", dtype=torch.int32)
    one = torch.ones(n, device="cuda")
    gap = (logits[:, 0].double() - logits[:, 1].double()) * (1 - 2 * ids)
    l = torch.nn.functional.logsigmoid(gap)
    d_other = -torch.sigmoid(-gap)  # dl/dz of the other token

    def check(got, coef):
        assert float((got["logprob"].double() - l).abs().max()) <= L_ABS + 2.0 ** -24 * float(l.abs().max())
        assert not bool(got["flags"].any())
        other = got["grad"].double().gather(1, 1 - ids[:, None].long())[:, 0]
        of_y = got["grad"].double().gather(1, ids[:, None].long())[:, 0]
        want = coef * d_other
        for x in (other - want, of_y + want):
            assert bool((x.abs() <= coef.abs() * (2.0 ** -21 + 2 * L_ABS) + 2.0 ** -23 * want.abs() + 1e-38).all())

    # ratio 1, advantage 1: the loss is -n / n
    got = pr.policy_loss(logits, ids, 1.0, one / n, one, l.float(), grad_scale=n)
    check(got, -(one / n).double() * n)
    assert abs(float(got["loss"]) + 1.0) <= 1e-5
    off = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    got = pr.preference_loss(logits, ids, 1.0, one, off, beta=1.0, grad_scale=n_pairs)
    h = l[0::2] - l[1::2]
    assert float((got["pair_logit"].double() - h).abs().max()) <= 2 * L_ABS + 2.0 ** -23 * float(h.abs().max())
    want = float(torch.nn.functional.softplus(-h).mean())
    assert abs(float(got["loss"]) - want) <= 2 * L_ABS + 2.0 ** -23
    check(got, torch.stack([-torch.sigmoid(-h), torch.sigmoid(-h)], 1).reshape(-1))


def test_many_rows_on_another_stream():
    """Calls on a stream of their own, with a workspace of the caller's filled with NaN, give the same results."""
    n, V = 700, 3001
    buf, logits, ids, T, w, A, old, ref = policy_inputs(n, V, torch.bfloat16, 0, 0, 9)
    cu = lambda x: torch.tensor(x, device="cuda")  # noqa: E731
    d, args = logits.cuda(), (cu(ids), cu(T), cu(w), cu(A), cu(old), cu(ref))
    off = torch.tensor([0, 100, 300, 300, 700], dtype=torch.int32, device="cuda")
    one = pr.policy_loss(d, *args, kl_coef=0.1)
    two = pr.preference_loss(d, *args[:3], off, args[5])
    L = _abi.lib()
    ws = [torch.full((int(b),), 255, dtype=torch.uint8, device="cuda") for b in
          (L.pr_policy_loss_workspace(_abi.PR_BF16, n, V), L.pr_preference_loss_workspace(_abi.PR_BF16, n, V, 2))]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = pr.policy_loss(d, *args, kl_coef=0.1, workspace=ws[0])
        b = pr.preference_loss(d, *args[:3], off, args[5], workspace=ws[1])
    side.synchronize()
    for x, y in ((one, a), (two, b)):
        for k in x:
            assert torch.equal(x[k], y[k]), k


def test_captured_in_a_graph():
    """A captured call gives the eager results on every replay, with new inputs in between."""
    n, V = 40, 5003
    buf, logits, ids, T, w, A, old, ref = policy_inputs(n, V, torch.bfloat16, 0, 0, 21)
    cu = lambda x: torch.tensor(x, device="cuda")  # noqa: E731
    d, args = logits.cuda(), (cu(ids), cu(T), cu(w), cu(A), cu(old), cu(ref))
    off = torch.tensor([0, 10, 40], dtype=torch.int32, device="cuda")
    call = lambda: (pr.policy_loss(d, *args, kl_coef=0.1), pr.preference_loss(d, *args[:3], off, args[5]))  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = call()
    for k in range(3):
        d.copy_(d.roll(k + 1, 1))
        eager = call()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip(eager, held):
            for key in x:
                assert torch.equal(x[key], y[key]), (k, key)


def test_refusals():
    dev = dict(device="cuda")
    z = torch.zeros(4, 32, **dev)
    ids = torch.zeros(4, dtype=torch.int32, **dev)
    f = torch.zeros(4, **dev)
    off = torch.tensor([0, 2, 4], dtype=torch.int32, **dev)
    for bad in (dict(logits=z.half()), dict(logits=z.cpu()), dict(logits=z.t()), dict(ids=ids.long()), dict(weight=f[:3]),
                dict(weight=f.double()), dict(advantage=f.cpu()), dict(old=f[::2]), dict(grad=z.bfloat16()),
                dict(grad=z[:, :16]), dict(ref=f[:2]), dict(logits=z[0])):
        a = dict(logits=z, ids=ids, weight=f, advantage=f, old=f, ref=None, grad=True, **{})
        a.update(bad)
        with pytest.raises((ValueError, TypeError)):
            pr.policy_loss(a["logits"], a["ids"], 1.0, a["weight"], a["advantage"], a["old"], a["ref"], grad=a["grad"])
    for opts in (dict(clip_low=1.5), dict(clip_low=-0.1), dict(clip_high=-1.0), dict(clip_high=math.nan),
                 dict(kl_coef=0.1), dict(grad_scale=math.inf)):
        with pytest.raises(pr.ProuterError):
            pr.policy_loss(z, ids, 1.0, f, f, f, **opts)
    wide = torch.zeros(5, 32, **dev)
    with pytest.raises(pr.ProuterError):  # the gradient may not overlap the logits other than in their place
        pr.policy_loss(wide[:4], ids, 1.0, f, f, f, grad=wide[1:])
    for bad_off in (off.long(), off[:2], off.cpu()):
        with pytest.raises(ValueError):
            pr.preference_loss(z, ids, 1.0, f, bad_off)
    for opts in (dict(beta=0.0), dict(beta=math.nan), dict(label_smoothing=1.1), dict(margin=math.inf)):
        with pytest.raises(pr.ProuterError):
            pr.preference_loss(z, ids, 1.0, f, off, **opts)


@pytest.mark.parametrize("n,V", [(1024, 1 << 22), (1, 1 << 26)])
def test_policy_long_rows(n, V):
    """Rows so long that a lane adds thousands of terms: the log-prob keeps the precision of the module docstring.
    All tokens but one share a logit, so that roundings do not average out."""
    logits = torch.empty(n, V, device="cuda")
    one = torch.ones(n, device="cuda")
    w = torch.zeros(n, device="cuda")
    w[0] = w[n - 1] = 1.0
    for z in (-0.3, -0.9, -1.1):
        for r in {0, n - 1}:
            logits[r] = z
            logits[r, 5] = 0.0
        ids = torch.full((n,), 5, dtype=torch.int32, device="cuda")
        want = -math.log1p((V - 1) * math.exp(float(np.float32(z))))
        for T, scale in ((1.0, 1.0), (0.5, 2.0)):
            l = want if T == 1.0 else -math.log1p((V - 1) * math.exp(2 * float(np.float32(z))))
            got = pr.policy_loss(logits, ids, T, w, one, one * l, grad=False)
            off = pr.preference_loss(logits, ids, T, w, torch.tensor([0, 0, n], dtype=torch.int32, device="cuda"),
                                     grad=False)
            for x in (got, off):
                near("logprob", x["logprob"][w != 0].cpu(), np.full(int(w.sum()), l), L_ABS, 2.0 ** -24)
