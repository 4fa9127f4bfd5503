"""The largest logits of rows, beam search's selection and the reordering of states: HIP path vs the fp64 oracle.

Tolerances: a log-prob is within 2e-6 (L, see the policy loss) of the exact one and rounded to float32 once (2^-24 of it);
tokens are exact. A beam's candidates are in the exact order among themselves; two beams' are when their scores are
further than 2 L + 2^-52 of them apart, and otherwise one of the two comes first.
"""

import numpy as np
import pytest
import torch

import paper_2608_28726_amd as pr
from oracle import beam as obeam
from oracle import distill as odist
from paper_2608_28726_amd import _abi
from tests.gpu_common import require_gpu
from tests.test_gpu_loss import L_ABS, make_rows, name_of, near, on_gpu, raw_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def cuda(x):
    return torch.tensor(np.ascontiguousarray(x), device="cuda")


def compare_top(g, o, what=""):
    torch.cuda.synchronize()
    assert np.array_equal(g["flags"].cpu().numpy(), o["flags"]), what
    assert np.array_equal(g["ids"].cpu().numpy(), o["ids"]), what
    # A log-prob below float32's range (-3.3e38 / 0.9) rounds to -inf.
    with np.errstate(over="ignore"):
        want = np.where(np.isinf(o["logprob"].astype(np.float32)), -np.inf, o["logprob"])
    near(what + "logprob", g["logprob"].cpu().numpy(), want, L_ABS)
    near(what + "lse", g["lse"].cpu().numpy(), o["lse"], L_ABS)


SHAPES = [
    # n, V, k, dtype, pad, start
    (1, 2, 1, torch.float32, 0, 0),
    (1, 2, 5, torch.bfloat16, 0, 1),
    (3, 7, 7, torch.bfloat16, 0, 1),
    (5, 9, 4, torch.float32, 3, 1),
    (17, 1000, 20, torch.float32, 5, 3),
    (9, 1537, 256, torch.bfloat16, 11, 5),
    (2, 255, 256, torch.float32, 0, 0),
    (4, 50257, 64, torch.bfloat16, 0, 0),
    (3, 50257, 256, torch.float32, 0, 2),
    (2, 151936, 64, torch.bfloat16, 0, 0),
    (2, 262144, 1, torch.float32, 0, 0),
    (2, 262147, 129, torch.bfloat16, 0, 7),
    (300, 4099, 17, torch.float32, 0, 0),
    (1500, 65, 8, torch.bfloat16, 0, 0),
    (300, 30011, 256, torch.bfloat16, 0, 1),
    (40, 30011, 12, torch.bfloat16, 0, 0),
    (520, 20000, 20, torch.float32, 0, 0),
]


@pytest.mark.parametrize("n,V,k,dtype,pad,start", SHAPES)
def test_top_against_the_oracle(n, V, k, dtype, pad, start):
    print("case", n, V, k, dtype, pad, start, flush=True)
    buf, logits, _, T, _ = make_rows(n, V, dtype, 31 * n + V + k, pad, start)
    g = pr.top_logits(on_gpu(buf, logits), k, cuda(T))
    compare_top(g, odist.top_logits(raw_of(logits), name_of(dtype), T, k))


def hard_rows(V, dtype, seed):
    """Rows whose largest logits lie or tie where a selection can go wrong."""
    rng = np.random.default_rng(seed)
    up = np.sort(rng.normal(0, 3, V))
    few = np.full(V, -np.inf)
    few[rng.permutation(V)[:10]] = rng.normal(0, 1, 10)
    low = np.full(V, -3.3e38)
    low[5:V // 2] = rng.normal(0, 1, V // 2 - 5)
    first, last = rng.normal(0, 1, V), rng.normal(0, 1, V)
    first[:200 if V > 400 else V // 4] += 50
    last[-(200 if V > 400 else V // 4):] += 50
    lane = rng.normal(0, 1, V)
    lane[::256 * 8] += 30
    lane[3::1024] += 20
    stuck = np.full(V, -np.inf)
    stuck[V // 3] = 1.0
    rows = [np.zeros(V), np.full(V, -2.5), up, up[::-1], np.round(rng.normal(0, 1, V)), few, low, first, last, lane, stuck,
            np.where(np.arange(V) % 2 == 0, 0.0, -0.0), np.repeat(up[::-8], 8)[:V] if V % 8 == 0 else up,
            np.where(rng.random(V) < 0.5, -np.inf, rng.normal(0, 0.01, V)), rng.normal(0, 1e-30, V),
            np.concatenate([np.full(V - V // 3, 1.0), rng.normal(0, 1, V // 3)])]
    z = torch.tensor(np.stack(rows))
    if dtype == torch.bfloat16:
        z = z.float().to(dtype)
    return z.to(dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [33, 4096, 50257])
@pytest.mark.parametrize("k", [1, 20, 64, 256])
def test_top_of_hard_rows(V, dtype, k):
    print("case", V, dtype, k, flush=True)
    z = hard_rows(V, dtype, V + k)
    T = np.linspace(0.5, 1.5, len(z)).astype(np.float32)
    o = odist.top_logits(raw_of(z), name_of(dtype), T, k)
    compare_top(pr.top_logits(z.cuda(), k, cuda(T)), o)
    # Among so many that each has a workgroup of its own
    many = 20
    g = pr.top_logits(z.repeat(many, 1).cuda(), k, cuda(np.tile(T, many)))
    compare_top(g, {name: np.concatenate([x] * many) for name, x in o.items()}, "many ")


@pytest.mark.parametrize("n", [8, 300])
def test_top_of_undefined_rows(n):
    z = torch.randn(n, 3001)
    z[0, 3000], z[1, 0], z[2], z[3, 5] = float("nan"), float("inf"), float("-inf"), float("-inf")
    T = np.ones(n, np.float32)
    T[4], T[5], T[6] = np.nan, 0.0, np.inf
    o = odist.top_logits(raw_of(z), "f32", T, 11)
    assert o["flags"][:8].tolist() == [1, 1, 1, 0, 4, 4, 4, 0]
    compare_top(pr.top_logits(z.cuda(), 11, cuda(T)), o)


def test_top_defaults_and_refusals():
    z = torch.randn(3, 100, device="cuda")
    a, b = pr.top_logits(z, 4), pr.top_logits(z, 4, torch.ones(3, device="cuda"))
    torch.cuda.synchronize()
    assert all(torch.equal(a[k], b[k]) for k in a)
    empty = pr.top_logits(z[:0], 4)
    assert empty["ids"].shape == (0, 4)
    for k in (0, 257):
        with pytest.raises(ValueError):
            pr.top_logits(z, k)
    with pytest.raises(ValueError):
        pr.top_logits(z.t(), 4)
    with pytest.raises(TypeError):
        pr.top_logits(z.half(), 4)
    with pytest.raises(ValueError):
        pr.top_logits(z, 4, torch.ones(2, device="cuda"))


# ---------------------------------------------------------------------------
# Selection

def compare_select(g, o, what=""):
    torch.cuda.synchronize()
    n_req, k = o["scores"].shape
    assert np.array_equal(g["flags"].cpu().numpy(), o["flags"]), what
    scores, parent, token, logprob = (g[x].cpu().numpy() for x in ("scores", "parent", "token", "logprob"))
    near(what + "scores", scores, o["scores"], 3 * L_ABS)
    for i in range(n_req):
        have = {(b, v): (s, l) for s, b, v, l in o["candidates"][i]}
        listed = o["candidates"][i]
        n = min(k, len(listed))
        assert (parent[i, n:] == -1).all() and (token[i, n:] == -1).all(), (what, i)
        assert np.isneginf(scores[i, n:]).all() and np.isneginf(logprob[i, n:]).all(), (what, i)
        got = list(zip(parent[i, :n].tolist(), token[i, :n].tolist()))
        assert len(set(got)) == n and all(c in have for c in got), (what, i)
        near(what + "logprob", logprob[i, :n], [have[c][1] for c in got], L_ABS)
        apart = 2 * L_ABS + 2.0 ** -40 * max([1.0] + [abs(c[0]) for c in listed[:n]])
        for j, c in enumerate(got):
            if c == listed[j][1:3]:
                continue
            # Another beam's candidate may only stand where the scores are that near.
            assert abs(have[c][0] - listed[j][0]) <= apart and c[0] != listed[j][1], (what, i, j, c, listed[j])


SELECT = [
    # n_req, B, V, k, dtype, pad, start
    (1, 1, 2, 1, torch.float32, 0, 0),
    (1, 1, 50, 60, torch.float32, 0, 0),
    (1, 4, 32000, 4, torch.float32, 0, 0),
    (1, 4, 151936, 8, torch.bfloat16, 0, 0),
    (3, 5, 1003, 7, torch.bfloat16, 3, 1),
    (2, 64, 517, 128, torch.float32, 0, 3),
    (1, 64, 4001, 256, torch.bfloat16, 0, 1),
    (70, 4, 6000, 8, torch.bfloat16, 0, 0),
    (2, 16, 50257, 16, torch.float32, 0, 0),
    (5, 3, 65, 33, torch.bfloat16, 0, 0),
    (400, 1, 300, 5, torch.float32, 0, 0),
    (33, 9, 257, 2, torch.bfloat16, 1, 0),
]


@pytest.mark.parametrize("n_req,B,V,k,dtype,pad,start", SELECT)
def test_select_against_the_oracle(n_req, B, V, k, dtype, pad, start):
    print("case", n_req, B, V, k, dtype, pad, start, flush=True)
    n = n_req * B
    buf, logits, _, T, rng = make_rows(n, V, dtype, 7 * n + V + k, pad, start)
    scores = rng.normal(-20, 2, (n_req, B)).astype(np.float32)
    done = rng.random((n_req, B)) < 0.2
    scores[rng.random((n_req, B)) < 0.1] = -np.inf
    d = on_gpu(buf, logits)
    raw, name = raw_of(logits), name_of(dtype)
    g = pr.beam_select(d, cuda(scores), cuda(T), k=k, done=cuda(done), done_token=5)
    compare_select(g, obeam.beam_select(raw, name, T, scores, k, done, 5))
    g = pr.beam_select(d, cuda(scores), cuda(T), k=k)
    compare_select(g, obeam.beam_select(raw, name, T, scores, k), "none done ")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n_req,B,V,k", [(1, 64, 50257, 128), (2, 64, 9000, 256), (3, 20, 20000, 256), (1, 1, 60000, 256),
                                         (60, 4, 3000, 256)])
def test_candidates_spread_unevenly(n_req, B, V, k, dtype):
    """Scores that leave most of the best to a few beams, or to all of them alike; beams of one token each beside them."""
    rng = np.random.default_rng([n_req, B, k])
    logits = torch.tensor(rng.normal(0, 1.5, (n_req * B, V)).astype(np.float32)).to(dtype)
    logits[::5, 1:] = -np.inf
    T = np.ones(n_req * B, np.float32)
    for spread in (0.0, 0.7, 6.0):
        scores = rng.normal(-20, spread, (n_req, B)).astype(np.float32)
        g = pr.beam_select(logits.cuda(), cuda(scores), cuda(T), k=k)
        o = obeam.beam_select(raw_of(logits), name_of(dtype), T, scores, k)
        torch.cuda.synchronize()
        best, parent, token = (g[x].cpu().numpy() for x in ("scores", "parent", "token"))
        near(f"spread {spread} scores", best, o["scores"], 3 * L_ABS)
        for i in range(n_req):
            listed = o["candidates"][i]
            n = min(k, len(listed))
            assert (parent[i, n:] == -1).all() and (token[i, n:] == -1).all()
            have = {(b, v): s for s, b, v, _ in listed}
            for j in range(n):  # candidates that near may stand in each other's place,
                assert abs(have[parent[i, j], token[i, j]] - listed[j][0]) <= 2 * L_ABS + 2.0 ** -40 * 100
            for b in range(B):  # but not those of one beam
                got = token[i, :n][parent[i, :n] == b].tolist()
                assert got == [v for _, c, v, _ in listed if c == b][:len(got)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("first", [0, 3])
def test_many_equal_candidates(first, dtype):
    """64 beams of equal logits: 16,384 candidates, all of one score, come out by beam and token."""
    B, V, k = 64, 300, 256
    scores = np.zeros((2, B), np.float32)
    scores[:, :first] = -np.inf
    g = pr.beam_select(torch.zeros(2 * B, V, dtype=dtype, device="cuda"), cuda(scores), k=k)
    torch.cuda.synchronize()
    assert (g["parent"] == first).all() and torch.equal(g["token"][1], torch.arange(k, dtype=torch.int32, device="cuda"))
    near("scores", g["scores"].cpu().numpy(), np.full((2, k), -np.log(V)), 3 * L_ABS)


def test_first_step_and_default_k():
    """At first only one beam exists: its best tokens, in order."""
    buf, logits, _, T, rng = make_rows(12, 700, torch.bfloat16, 2)
    scores = np.full((3, 4), -np.inf, np.float32)
    scores[:, 0] = 0.0
    g = pr.beam_select(logits.cuda(), cuda(scores), cuda(T))
    top = pr.top_logits(logits.cuda(), 4, cuda(T))
    torch.cuda.synchronize()
    assert (g["parent"] == 0).all() and torch.equal(g["token"], top["ids"][::4])
    assert torch.equal(g["scores"], top["logprob"][::4]) and torch.equal(g["logprob"], top["logprob"][::4])


@pytest.mark.parametrize("k", [3, 64, 256])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_select_among_equals(k, dtype):
    """Equal beams, equal logits and equal scores come out by beam and token; scores that swallow all log-probs too."""
    V, B = 300, 6
    same = torch.zeros(B, V, dtype=dtype)
    twice = torch.randn(1, V).to(dtype).repeat(B, 1)
    lost = torch.randn(B, V).to(dtype)
    rows = torch.cat([same, twice, lost, lost])
    T = np.ones(4 * B, np.float32)
    scores = np.zeros((4, B), np.float32)
    scores[2] = -3e38  # any log-prob is lost beside it
    scores[3] = [-1e30, -2.0, -2.0, -1e30, -2.0, -np.inf]
    g = pr.beam_select(rows.cuda(), cuda(scores), cuda(T), k=k)
    torch.cuda.synchronize()
    parent, token = g["parent"].cpu().numpy(), g["token"].cpu().numpy()
    assert parent[0].tolist() == [i // V for i in range(k)] and token[0].tolist() == [i % V for i in range(k)]
    order = np.lexsort((np.arange(V), -lost.double().numpy()[0]))
    assert (parent[2] == 0).all() and token[2].tolist() == order[:k].tolist()
    o = obeam.beam_select(raw_of(rows), name_of(dtype), T, scores, k)
    for i in (0, 1, 3):
        assert parent[i].tolist() == o["parent"][i].tolist() and token[i].tolist() == o["token"][i].tolist(), i


def test_beams_that_are_undefined():
    n_req, B, V = 2, 5, 100
    z = torch.randn(n_req * B, V)
    z[1, 7], z[2], z[7] = float("nan"), float("-inf"), float("nan")
    T = np.ones(n_req * B, np.float32)
    T[3] = 0.0
    scores = np.zeros((n_req, B), np.float32)
    scores[1, 0], scores[1, 1], scores[1, 2] = np.nan, np.inf, -np.inf
    g = pr.beam_select(z.cuda(), cuda(scores), cuda(T), k=6)
    o = obeam.beam_select(raw_of(z), "f32", T, scores, 6)
    assert o["flags"].tolist() == [0, 1, 1, 4, 0, 1, 1, 16, 0, 0]
    compare_select(g, o)
    nothing = pr.beam_select(z.cuda(), torch.full((2, 5), float("-inf"), device="cuda"), 1.0)
    torch.cuda.synchronize()
    assert (nothing["parent"] == -1).all() and (nothing["token"] == -1).all() and torch.isinf(nothing["scores"]).all()
    ended = pr.beam_select(z.cuda(), cuda(np.arange(10, dtype=np.float32).reshape(2, 5)), 1.0, k=3,
                           done=torch.ones(2, 5, dtype=torch.uint8, device="cuda"), done_token=-9)
    torch.cuda.synchronize()
    assert ended["parent"].tolist() == [[4, 3, 2]] * 2 and (ended["token"] == -9).all()
    assert ended["scores"].tolist() == [[4, 3, 2], [9, 8, 7]] and (ended["logprob"] == 0).all()


def test_select_refusals():
    z, s = torch.randn(6, 50, device="cuda"), torch.zeros(2, 3, device="cuda")
    for kw in (dict(scores=s.view(6)), dict(scores=s.double()), dict(scores=torch.zeros(2, 2, device="cuda")),
               dict(scores=s.t()), dict(k=0), dict(k=257), dict(done=torch.zeros(6, dtype=torch.bool, device="cuda")),
               dict(done=torch.zeros(2, 3, device="cuda")), dict(done_token=1 << 31), dict(scores=s.cpu()),
               dict(temperature=torch.ones(2, 3, device="cuda"))):
        with pytest.raises(ValueError):
            pr.beam_select(z, **{"scores": s, **kw})
    with pytest.raises(ValueError):
        pr.beam_select(torch.randn(65, 50, device="cuda"), torch.zeros(1, 65, device="cuda"))
    assert pr.beam_select(z[:0], s[:0])["token"].shape == (0, 3)


def test_repeatable_captured_and_on_another_stream():
    cases = []
    for n_req, B, V, k in ((1, 4, 50257, 8), (80, 4, 3000, 4), (3, 33, 700, 66)):
        buf, logits, _, T, rng = make_rows(n_req * B, V, torch.bfloat16, V)
        cases.append((logits.cuda(), cuda(rng.normal(-5, 1, (n_req, B)).astype(np.float32)), cuda(T), k))
    calls = [lambda x=x: pr.beam_select(*x) for x in cases] + [lambda x=x: pr.top_logits(x[0], x[3], x[2]) for x in cases]
    want = [f() for f in calls]
    again = [f() for f in calls]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = [f() for f in calls]
    torch.cuda.synchronize()
    for a, b, c in zip(want, again, other):
        assert all(torch.equal(a[k], b[k]) and torch.equal(a[k], c[k]) for k in a)
    graphs = []
    for f in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = f()
        graphs.append((g, out))
    for _ in range(3):
        for (g, out), w in zip(graphs, want):
            for t in out.values():
                t.fill_(3)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(out[k], w[k]) for k in w)


def test_workspaces_of_the_caller():
    buf, logits, _, T, rng = make_rows(8, 30000, torch.float32, 5)
    d, t = logits.cuda(), cuda(T)
    s = cuda(rng.normal(0, 1, (2, 4)).astype(np.float32))
    L = _abi.lib()
    ws = torch.full((max(L.pr_top_logits_workspace(0, 8, 30000, 9), L.pr_beam_select_workspace(0, 2, 4, 30000, 9), 16),), 255,
                    dtype=torch.uint8, device="cuda")
    for f in (lambda **kw: pr.top_logits(d, 9, t, **kw), lambda **kw: pr.beam_select(d, s, t, k=9, **kw)):
        a, b = f(), f(workspace=ws)
        torch.cuda.synchronize()
        assert all(torch.equal(a[k], b[k]) for k in a)


# ---------------------------------------------------------------------------
# Reordering

def parents(n_req, B, seed, out=0.1):
    rng = np.random.default_rng(seed)
    p = rng.integers(0, B, (n_req, B)).astype(np.int32)
    p[rng.random((n_req, B)) < out] = rng.choice([-1, B, -2 ** 31, 2 ** 31 - 1])
    return p


def bytes_of(shape, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    size = torch.empty(0, dtype=dtype).element_size()
    n = int(np.prod(shape))
    return torch.randint(0, 256, (n * size,), dtype=torch.uint8, generator=g).view(dtype).view(shape)


@pytest.mark.parametrize("n_req,B", [(1, 1), (1, 2), (1, 4), (7, 3), (3, 8), (5, 9), (2, 32), (3, 33), (2, 64), (200, 4)])
def test_reorder(n_req, B):
    print("case", n_req, B, flush=True)
    n = n_req * B
    shapes = [((n,), torch.int32), ((n, 1), torch.uint8), ((n, 3), torch.uint8), ((n, 15), torch.uint8), ((n, 16), torch.uint8),
              ((n, 17), torch.uint8), ((n_req, B, 5, 7), torch.bfloat16), ((n, 33), torch.float32), ((n, 0), torch.float32),
              ((n, 257, 9), torch.int64 if n < 300 else torch.int16)]
    before = [bytes_of(s, t, i) for i, (s, t) in enumerate(shapes)]
    p = parents(n_req, B, n)
    states = [x.cuda() for x in before]
    pr.beam_reorder(states, cuda(p))
    torch.cuda.synchronize()
    for x, y in zip(before, states):
        rows = x.reshape(n, -1).view(torch.uint8) if x.numel() else x
        got = y.cpu().reshape(n, -1).view(torch.uint8) if x.numel() else y.cpu()
        assert np.array_equal(got.numpy(), obeam.reorder(rows.numpy(), p)), (x.shape, x.dtype)


def test_reorder_of_rows_apart_and_side_by_side():
    """Rows that lie apart leave what is between them; two states in one stride; rows at odd addresses."""
    n_req, B = 3, 4
    p = parents(n_req, B, 5)
    buf = bytes_of((12, 101), torch.uint8, 1)
    d = buf.cuda()
    pr.beam_reorder([d[:, 3:20], d[:, 20:97]], cuda(p))
    torch.cuda.synchronize()
    want = buf.clone().numpy()
    want[:, 3:97] = obeam.reorder(want[:, 3:97], p)
    assert np.array_equal(d.cpu().numpy(), want)
    one = bytes_of((12, 50), torch.float32, 2)
    d = one.cuda()
    pr.beam_reorder(d[:, 1:], cuda(p))
    torch.cuda.synchronize()
    want = one.clone().view(torch.int32).numpy()
    want[:, 1:] = obeam.reorder(want[:, 1:], p)
    assert np.array_equal(d.cpu().view(torch.int32).numpy(), want)


def test_reorder_many_states_and_long_rows():
    n_req, B = 2, 4
    p = parents(n_req, B, 9)
    before = [bytes_of((8, 5 + i), torch.int16, i) for i in range(201)] + [bytes_of((8, 1_500_001), torch.int16, 999)]
    states = [x.cuda() for x in before]
    pr.beam_reorder(states, cuda(p))
    torch.cuda.synchronize()
    for x, y in zip(before, states):
        assert np.array_equal(y.cpu().numpy(), obeam.reorder(x.numpy(), p))


def test_reorder_refusals():
    p = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    x = torch.zeros(6, 10, device="cuda")
    for bad in (x[:5], x.cpu(), x.t(), torch.zeros(6, 10, 2, device="cuda")[:, :, 0], x[:, None].expand(6, 2, 10)[:, :, :5],
                torch.zeros(1, 10, device="cuda").expand(6, 10), torch.zeros(3, 2, 10, device="cuda").transpose(0, 1),
                torch.zeros(6, 4, 8, device="cuda")[:, :, :4]):
        with pytest.raises(ValueError):
            pr.beam_reorder([bad], p)
    with pytest.raises(pr.ProuterError):
        pr.beam_reorder([x, x], p)
    with pytest.raises(pr.ProuterError):
        pr.beam_reorder([x[:, :6], x[:, 5:]], p)
    for bad in (p.long(), p.view(6), p.t(), p.cpu(), torch.zeros(1, 65, dtype=torch.int32, device="cuda")):
        with pytest.raises(ValueError):
            pr.beam_reorder([torch.zeros(65, 2, device="cuda")], bad)
    pr.beam_reorder([], p)
    pr.beam_reorder([torch.zeros(0, 3, device="cuda")], p[:0])


def test_reorder_captured():
    n_req, B = 5, 4
    before = [bytes_of((20, 700), torch.int32, 3), bytes_of((20, 3), torch.int16, 4)]
    p = parents(n_req, B, 11)
    states, parent = [x.cuda() for x in before], torch.zeros(n_req, B, dtype=torch.int32, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pr.beam_reorder(states, parent)
    for step in range(4):  # the parents are read at each replay
        p = parents(n_req, B, step)
        for x, y in zip(states, before):
            x.copy_(y)
        parent.copy_(torch.tensor(p))
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip(before, states):
            assert np.array_equal(y.cpu().numpy(), obeam.reorder(x.numpy(), p))


@pytest.mark.parametrize("max_len", [0, 9, 40])
def test_stream_reorder(max_len):
    """A beam's slot takes its parent's history: the verdicts are those of a stream that saw that history alone."""
    n_req, B, V, steps = 3, 4, 300, 12
    n = n_req * B
    slots = torch.tensor(np.random.default_rng(1).permutation(20)[:n].astype(np.int32), device="cuda")
    st, ref = pr.StreamState(20, max_len, q=0.3), pr.StreamState(20, max_len, q=0.3)
    gen = torch.Generator(device="cuda").manual_seed(5)
    history = [[] for _ in range(n)]  # each beam's (logit row, token) so far
    for t in range(steps):
        logits = torch.randn(n, V, device="cuda", generator=gen) * 3
        ids = torch.randint(0, V, (n,), device="cuda", generator=gen, dtype=torch.int32)
        st.step(logits, slots, ids, 1.0)
        for r in range(n):
            history[r].append((logits[r], ids[r]))
        p = parents(n_req, B, 100 + t)
        st.reorder(slots.view(n_req, B), cuda(p))
        history = [list(history[i * B + q]) if 0 <= q < B else history[i * B + b]
                   for i in range(n_req) for b, q in enumerate(p[i].tolist())]
    for t in range(steps):
        ref.step(torch.stack([h[t][0] for h in history]), slots, torch.stack([h[t][1] for h in history]), 1.0)
    a, b = st.finish(slots, 0.2), ref.finish(slots, 0.2)
    torch.cuda.synchronize()
    for k in a:
        x, y = a[k].cpu().numpy(), b[k].cpu().numpy()
        assert np.array_equal(x, y, equal_nan=x.dtype.kind == "f"), k
    st.close()
    ref.close()


def test_stream_reorder_leaves_other_slots():
    st = pr.StreamState(6, 8)
    z = torch.randn(6, 50, device="cuda")
    ids = torch.zeros(6, dtype=torch.int32, device="cuda")
    every = torch.arange(6, dtype=torch.int32, device="cuda")
    f = st.step(z, every, ids, 1.0, want_features=True)
    slots = torch.tensor([[1, 99], [-1, 3], [4, 2]], dtype=torch.int32, device="cuda")
    st.reorder(slots, torch.tensor([[1, 0], [1, 0], [1, 1]], dtype=torch.int32, device="cuda"))
    out = st.finish(every, 0.0)
    torch.cuda.synchronize()
    want = f["maxprob"].clone()
    want[4] = f["maxprob"][2]
    assert torch.equal(out["mean"][:, 1], want) and (out["count"] == 1).all()
    with pytest.raises(ValueError):
        st.reorder(slots.view(-1), torch.zeros(3, 2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        st.reorder(slots.long(), torch.zeros(3, 2, dtype=torch.int32, device="cuda"))
    st.close()
