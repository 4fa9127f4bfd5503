"""Top logits, beam selection and the distillation loss at the limits: more elements than 32 bits count, the longest
row, more rows than a kernel lists, calls that overlap."""

import math

import numpy as np
import pytest
import torch

import paper_2608_28726_amd as pr
from tests.gpu_common import require_gpu

pytestmark = pytest.mark.gpu

LONGEST = 2 ** 31 - 1


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()
    yield
    torch.cuda.empty_cache()


def rows(n, V, dtype, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    z = torch.empty(n, V, dtype=dtype, device="cuda")
    for a in range(0, n, 1024):
        z[a:a + 1024] = torch.empty(min(1024, n - a), V, device="cuda").normal_(generator=g).mul_(2.0)
    return z, g


def same(a, b, names=None):
    torch.cuda.synchronize()
    for k in names or a:
        assert torch.equal(a[k], b[k]), k


def test_more_elements_than_32_bits_count():
    n, V, k = 17000, 151936, 20
    z, g = rows(n, V, torch.bfloat16, 1)
    last = slice(n - 64, n)
    top = pr.top_logits(z, k)
    few = pr.top_logits(z[last], k)
    torch.cuda.synchronize()
    assert torch.equal(top["ids"][last], few["ids"])
    # (64 rows are summed in parts: their log-probs agree to the sums' rounding, 2e-6 each.)
    assert (top["logprob"][last] - few["logprob"]).abs().max().item() <= 4e-6 + 2.0 ** -23 * 30
    scores = torch.zeros(n // 4, 4, device="cuda")
    select = pr.beam_select(z, scores)
    some = pr.beam_select(z[n - 4096:].clone(), scores[:1024])  # as many rows as are not summed in parts
    same({x: select[x][-1024:] for x in ("scores", "parent", "token", "logprob")}, some, ("scores", "parent", "token", "logprob"))
    w = torch.full((n,), 1.0 / n, device="cuda")
    w[torch.rand(n, device="cuda", generator=g) < 0.2] = 0.0
    whole = pr.distill_loss(z, top["ids"], top["logprob"], 0.9, w)
    part = pr.distill_loss(z[n - 4096:].clone(), top["ids"][n - 4096:], top["logprob"][n - 4096:], 0.9, w[n - 4096:])
    same({x: whole[x][n - 4096:] for x in ("token_loss", "mass", "flags", "grad")}, part, ("token_loss", "mass", "flags", "grad"))


def test_more_rows_than_are_listed():
    """66,000 held rows, dealt out by row; the same rows in two calls, dealt out by rank."""
    n, V, k = 66_000, 28_000, 7
    z, g = rows(n, V, torch.bfloat16, 2)
    top = pr.top_logits(z, k)
    w = torch.rand(n, device="cuda", generator=g)
    w[torch.rand(n, device="cuda", generator=g) < 0.3] = 0.0
    w[:600] = 0.0
    whole = pr.distill_loss(z, top["ids"], top["logprob"], 1.2, w)
    for part in (slice(0, n // 2), slice(n // 2, n)):
        half = pr.distill_loss(z[part], top["ids"][part], top["logprob"][part], 1.2, w[part])
        same({x: whole[x][part] for x in ("token_loss", "mass", "flags", "grad")}, half, ("token_loss", "mass", "flags", "grad"))
    want = (w.double() * whole["token_loss"].double()).sum().item()
    # The row terms are rounded to float32 here, 2^-24 of each.
    assert abs(whole["loss"].item() - want) <= 2.0 ** -22 * (w * whole["token_loss"].abs()).double().sum().item()


def test_the_longest_row():
    """2^31 - 1 logits: zeros beside three larger ones, at both ends and in the middle."""
    z = torch.zeros(1, LONGEST, dtype=torch.bfloat16, device="cuda")
    at, height = [LONGEST - 1, 0, 1_500_000_001], [20.0, 19.0, 18.0]
    for i, h in zip(at, height):
        z[0, i] = h
    S = (LONGEST - 3) + sum(map(math.exp, height))
    lse = math.log(S)
    top = pr.top_logits(z, 5)
    torch.cuda.synchronize()
    assert top["ids"][0].tolist() == at + [1, 2]
    assert abs(top["lse"].item() - lse) <= 2e-6 + 2.0 ** -23 * lse
    want = np.array([h - lse for h in height] + [-lse] * 2)
    assert np.abs(top["logprob"][0].cpu().double().numpy() - want).max() <= 2e-6 + 2.0 ** -23 * lse
    select = pr.beam_select(z, torch.zeros(1, 1, device="cuda"), k=4)
    torch.cuda.synchronize()
    assert select["token"][0].tolist() == at + [1]
    # The student's own largest as the teacher's, with other probabilities and a token among the zeros.
    ids = torch.tensor([at + [LONGEST - 2]], dtype=torch.int32, device="cuda")
    q = np.array([0.4, 0.3, 0.1, 0.05])
    logq = torch.tensor(np.log(q)[None].astype(np.float32), device="cuda")
    q = np.exp(logq[0].cpu().double().numpy())
    out = pr.distill_loss(z, ids, logq, 1.0, torch.ones(1, device="cuda"))
    torch.cuda.synchronize()
    p = np.exp(np.array(height + [0.0]) - lse)
    P, Q = p.sum(), q.sum()
    loss = (q * (np.log(q) - np.log(p))).sum() + (1 - Q) * math.log((1 - Q) / (1 - P))
    assert abs(out["loss"].item() - loss) <= 4e-6 + 2.0 ** -23 * loss
    for i, (v, pv, qv) in enumerate(zip(at + [LONGEST - 2], p, q)):
        g = out["grad"][0, v].item()
        assert abs(g - (pv - qv)) <= 6e-6 + 2.0 ** -8 * 1.01 * abs(pv - qv), i
    other = (Q - P * (1 - Q) / (1 - P)) * math.exp(-lse)
    mid = out["grad"][0, 2 ** 30 - 5:2 ** 30 + 5].double()
    assert (mid - other).abs().max().item() <= abs(other) * (2.0 ** -8 * 1.01 + 2e-5)


def test_calls_that_overlap():
    """The same operators on two streams at once, on inputs of their own."""
    cases = []
    for seed, (n, V) in enumerate(((300, 30011), (8, 151936), (300, 30011), (8, 151936))):
        z, g = rows(n, V, torch.float32, seed)
        cases.append((z, torch.randn(n // 4, 4, device="cuda", generator=g), torch.full((n,), 1.0 / n, device="cuda")))

    def all_of(z, scores, w):
        top = pr.top_logits(z, 30, 0.8)
        best = pr.beam_select(z, scores, 0.8, k=9)
        loss = pr.distill_loss(z, top["ids"], top["logprob"], 1.1, w)
        moved = z.clone()
        pr.beam_reorder([moved], best["parent"][:, :4].contiguous())
        return {**{"t" + k: v for k, v in top.items()}, **{"b" + k: v for k, v in best.items()}, **loss, "moved": moved}

    want = [all_of(*c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = []
        for i, c in enumerate(cases):
            with torch.cuda.stream(streams[i % 2]):
                got.append(all_of(*c))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            same(a, b)
