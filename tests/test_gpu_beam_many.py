"""Top logits and beam selection over more rows than a launch of wide workgroups holds (2^31 threads)."""

import numpy as np
import pytest
import torch

import paper_2608_28726_amd as pr
from oracle import beam as obeam
from oracle import distill as odist
from tests.gpu_common import require_gpu
from tests.test_gpu_beam import compare_select, compare_top
from tests.test_gpu_loss import raw_of

pytestmark = pytest.mark.gpu

MANY = 2 ** 23


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()
    yield
    torch.cuda.empty_cache()


def rows(n, V, dtype, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty(n, V, dtype=torch.float32, device="cuda").normal_(generator=g).to(dtype), g


@pytest.mark.parametrize("n,k", [(MANY, 65), (MANY + 37, 65), (MANY + 37, 2)])
def test_top_of_more_rows_than_a_launch_holds(n, k):
    print("case", n, k, flush=True)
    V = 3
    z, g = rows(n, V, torch.bfloat16, k)
    T = torch.rand(n, device="cuda", generator=g) + 0.5
    top = pr.top_logits(z, k, T)
    torch.cuda.synchronize()
    order = torch.sort(z.float(), dim=1, descending=True, stable=True).indices[:, :k]  # equal ones by lower index
    for a in range(0, n, 1 << 21):  # all rows: none is left unwritten
        part = slice(a, a + (1 << 21))
        assert torch.equal(top["ids"][part, :V], order[part].int()), a
        assert (top["ids"][part, V:] == -1).all() and torch.isneginf(top["logprob"][part, V:]).all(), a
        assert (top["flags"][part] == 0).all() and top["lse"][part].isfinite().all(), a
    for part in (slice(0, 40), slice(n // 2 - 20, n // 2 + 20), slice(n - 60, n)):
        o = odist.top_logits(raw_of(z[part].cpu()), "bf16", T[part].cpu().numpy(), k)
        compare_top({name: x[part] for name, x in top.items()}, o, str(part))


@pytest.mark.parametrize("k", [65, 3])
def test_select_of_as_many_beams_as_are_allowed(k):
    """2^23 beams against the same requests in two calls, each of one launch; the first and last against the oracle."""
    V, B = 3, 64
    n_req = MANY // B
    z, g = rows(MANY, V, torch.bfloat16, k)
    scores = torch.empty(n_req, B, device="cuda").normal_(generator=g).mul_(2.0)
    done = torch.rand(n_req, B, device="cuda", generator=g) < 0.1
    whole = pr.beam_select(z, scores, 0.9, k, done, 7)
    half = n_req // 2
    for part in (slice(0, half), slice(half, n_req)):
        some = pr.beam_select(z[part.start * B:part.stop * B], scores[part], 0.9, k, done[part], 7)
        torch.cuda.synchronize()
        for name in ("scores", "parent", "token", "logprob"):
            assert torch.equal(whole[name][part], some[name]), (name, part)
        assert torch.equal(whole["flags"].view(n_req, B)[part].reshape(-1), some["flags"])
    for part in (slice(0, 2), slice(n_req - 2, n_req)):
        raw, T = raw_of(z[part.start * B:part.stop * B].cpu()), np.full(2 * B, 0.9, np.float32)
        o = obeam.beam_select(raw, "bf16", T, scores[part].cpu().numpy(), k, done[part].cpu().numpy(), 7)
        got = {name: x[part] for name, x in whole.items() if name != "flags"}
        got["flags"] = whole["flags"].view(n_req, B)[part].reshape(-1)
        compare_select(got, o)
    with pytest.raises(pr.ProuterError):
        pr.beam_select(torch.zeros(MANY + 1, 2, dtype=torch.bfloat16, device="cuda"), torch.zeros(MANY + 1, 1, device="cuda"))


def test_distillation_of_more_rows_than_a_launch_holds():
    """2^23 + 37 rows, whose sums take two launches and whose gradients 257, against the same rows in two calls; the
    last ones against the oracle."""
    n, V, k = MANY + 37, 5, 2
    z, g = rows(n, V, torch.float32, 9)
    top = pr.top_logits(z.flip(1).contiguous(), k, 1.0)
    w = torch.rand(n, device="cuda", generator=g)
    w[torch.rand(n, device="cuda", generator=g) < 0.2] = 0.0
    T = torch.rand(n, device="cuda", generator=g) + 0.5
    whole = pr.distill_loss(z, top["ids"], top["logprob"], T, w)
    half = n // 2
    for part in (slice(0, half), slice(half, n)):
        some = pr.distill_loss(z[part], top["ids"][part], top["logprob"][part], T[part], w[part])
        torch.cuda.synchronize()
        for name in ("token_loss", "mass", "flags", "grad"):
            assert torch.equal(whole[name][part], some[name]), (name, part)
    part = slice(n - 50, n)
    raw = raw_of(z[part].cpu())
    o = odist.distill_loss(raw, "f32", *(x[part].cpu().numpy() for x in (top["ids"], top["logprob"], T, w)))
    # A row's loss and gradient are off by the log-probs' 2e-6 and a rounding (its terms are at most a few units).
    assert np.abs(whole["token_loss"][part].cpu().numpy() - o["token_loss"]).max() <= 1e-5
    assert np.abs(whole["grad"][part].cpu().numpy() - o["grad"]).max() <= 1e-5
