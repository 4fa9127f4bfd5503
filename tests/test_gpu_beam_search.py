"""Beam search, the verifier, a teacher's top logits and the distillation step as they are used together."""

import math

import numpy as np
import pytest
import torch

import paper_2608_28726_amd as pr
from oracle import beam as obeam
from oracle import distill as odist
from paper_2608_28726_amd import beam_search as bs
from paper_2608_28726_amd import post_train as pt
from paper_2608_28726_amd import workloads as wl
from tests.gpu_common import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def table(n_req, V, length, seed, spread=3.0):
    """Logits of step t after token v: a table, so that what follows a beam is known."""
    rng = np.random.default_rng(seed)
    first = rng.normal(0, spread, (n_req, V)).astype(np.float32)
    after = rng.normal(0, spread, (length, V, V)).astype(np.float32)
    return first, after


def plain_search(first, after, n_req, B, length, T, end):
    """The same search with the oracle's steps; also each beam's rows."""
    V = first.shape[1]
    scores = np.full((n_req, B), -np.inf, np.float32)
    scores[:, 0] = 0
    tokens = np.full((n_req * B, length), -1)
    rows = np.zeros((n_req * B, length, V), np.float32)
    done = np.zeros((n_req, B), bool)
    last = np.zeros(n_req * B, int)
    for t in range(length):
        z = np.repeat(first, B, 0) if t == 0 else after[t][np.maximum(last, 0)]
        o = obeam.beam_select(z, "f32", np.full(n_req * B, T, np.float32), scores, B, done if end is not None else None)
        scores = o["scores"].astype(np.float32)
        parent = o["parent"]
        tokens, rows = obeam.reorder(tokens, parent), obeam.reorder(rows, parent)
        rows[:, t] = obeam.reorder(z, parent)
        done = obeam.reorder(done.reshape(-1), parent).reshape(n_req, B)
        last = o["token"].reshape(-1)
        tokens[:, t] = last
        if end is not None:
            done |= (last == end).reshape(n_req, B)
    return scores, tokens.reshape(n_req, B, length), rows, done


@pytest.mark.parametrize("end", [None, 3])
@pytest.mark.parametrize("n_req,B,V,length", [(1, 1, 10, 4), (3, 4, 40, 6), (5, 7, 33, 5), (2, 6, 4, 5)])
def test_search_against_the_oracle(n_req, B, V, length, end):
    """Tokens, scores and the verifier's summaries of every beam (V = 4: at first there are fewer tokens than beams)."""
    T = 0.9
    first, after = table(n_req, V, length, 100 * V + length)
    d_first, d_after = torch.tensor(first).cuda(), torch.tensor(after).cuda()
    stream = pr.StreamState(n_req * B, length)
    slots = torch.arange(n_req * B, dtype=torch.int32, device="cuda").view(n_req, B)

    def next_logits(t, tokens):
        if t == 0:
            return d_first.repeat_interleave(B, 0)
        return d_after[t][tokens.clamp(min=0).long()]

    mark = torch.zeros(n_req * B, length, device="cuda")  # a state of each beam: its tokens once more

    def marked(t, tokens):
        if tokens is not None:
            mark[:, t - 1] = tokens.float()
        return next_logits(t, tokens)

    out = bs.beam_search(marked, n_req, B, length, T, end, [mark], stream, slots)
    scores, tokens, rows, done = plain_search(first, after, n_req, B, length, T, end)
    torch.cuda.synchronize()
    assert np.array_equal(out["tokens"].cpu().numpy(), tokens)
    assert np.array_equal(out["done"].cpu().numpy(), done)
    got = out["scores"].cpu().numpy()
    assert np.array_equal(np.isinf(got), np.isinf(scores))
    # Each step adds a log-prob within 2e-6 and rounds the sum twice (here and in the oracle's float32).
    fin = np.isfinite(scores)
    assert (np.abs(got[fin] - scores[fin]) <= length * (2e-6 + 2 * 2.0 ** -24 * np.abs(scores[fin]))).all()
    live = np.isfinite(scores).reshape(-1)
    assert np.array_equal(mark.cpu().numpy()[live, :length - 1], tokens.reshape(-1, length)[live, :length - 1])
    # The verifier has seen each beam's rows and tokens, up to its end, and nothing else.
    have = stream.finish(slots.view(-1), 0.0)
    torch.cuda.synchronize()
    for r in np.flatnonzero(live):
        seen = [t for t in range(length) if tokens.reshape(-1, length)[r, t] >= 0]
        assert have["count"][r].item() == len(seen)
        z, ids = torch.tensor(rows[r, seen]).cuda(), torch.tensor(tokens.reshape(-1, length)[r, seen].astype(np.int32)).cuda()
        alone = pr.request_aggregate(pr.token_features(z, ids, T), torch.tensor([0, len(seen)], dtype=torch.int32,
                                                                                device="cuda"))
        torch.cuda.synchronize()
        for name in ("mean", "min", "quant", "score"):
            a, b = have[name][r].cpu().double().numpy(), alone[name][0].cpu().double().numpy()
            assert np.all(np.abs(a - b) <= 1e-5 + 1e-4 * np.abs(b)), (r, name)
    stream.close()


def test_the_distill_step_takes_the_oracles_gradient():
    """One step of the example: what the layer is given is the oracle's gradient of these rows."""
    vocab, width, length = 500, 32, 4
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    hidden = torch.empty(8 * length, width, device="cuda").normal_(generator=g).bfloat16()
    rows, top = pt._teacher(hidden, vocab, length, seed=5)
    assert rows.shape == (8 * length, width) and top["ids"].shape == (8 * length, pt.TOP)
    layer = pt.OutputLayer(vocab, width, 32, 7, "cuda")
    weight = torch.full((len(rows),), 1.0 / len(rows), device="cuda")
    logits = layer.logits(rows)
    raw = wl.to_host_raw(logits.cpu())
    given = []
    layer.step = lambda h, grad, lr: given.append((h.clone(), grad.float().cpu().numpy()))
    loss, agree = pt._distill_step(layer, rows, top, weight, 0.1)
    o = odist.distill_loss(raw, "bf16", top["ids"].cpu().numpy(), top["logprob"].cpu().numpy(),
                           np.full(len(rows), pt.TEMPERATURE, np.float32), weight.cpu().numpy())
    assert len(given) == 1 and torch.equal(given[0][0], rows)
    # The element tolerance of the loss's own test: 6e-6 of the coefficient and half a bfloat16 step.
    tol = 6e-6 * np.abs(o["coef"])[:, None] + (2.0 ** -8 * 1.01 + 2.0 ** -22) * np.abs(o["grad"])
    assert (np.abs(given[0][1] - o["grad"]) <= tol).all()
    assert abs(loss.item() - o["loss"]) <= 4e-6 + 2.0 ** -23 * abs(o["loss"])
    assert 0.0 <= float(agree) <= 1.0


def test_examples_run(capsys):
    out = pt.post_train("distill", steps=5, vocab=512, requests=16, length=4)
    assert len(out["loss"]) == 5 and all(math.isfinite(v) for v in out["loss"] + out["reward"])
    assert 0.0 <= out["reward_after"] <= 1.0
    assert bs.main(["5", "3", "4"]) == 0
    assert "answers ship" in capsys.readouterr().out
    assert pt.main(["distill", "2"]) == 0


def test_beams_that_cease_to_exist():
    """Rows that are NaN leave a request without candidates: no tokens, no end, and the other request goes on."""
    n_req, B, V, length = 2, 3, 20, 4
    first, after = table(n_req, V, length, 5)
    d_first, d_after = torch.tensor(first).cuda(), torch.tensor(after).cuda()

    def next_logits(t, tokens):
        if t == 0:
            return d_first.repeat_interleave(B, 0)
        z = d_after[t][tokens.clamp(min=0).long()]
        if t == 2:
            z[:B] = math.nan
        return z

    out = bs.beam_search(next_logits, n_req, B, length, 1.0, end=None)
    assert (out["scores"][0] == -math.inf).all() and (out["tokens"][0] == -1).all() and not out["done"].any()
    scores, tokens, _, _ = plain_search(first[1:], after, 1, B, length, 1.0, None)
    assert np.array_equal(out["tokens"][1].cpu().numpy(), tokens[0])


@pytest.mark.parametrize("max_len", [0, 4])
def test_the_verifier_of_beams_that_cease_to_exist(max_len):
    """A request that loses its candidates, one that goes on, and one that never had as many as beams: the verifier has
    seen the beams that are there, and no answer of the others ships."""
    n_req, B, V, length = 3, 3, 20, 4
    first, after = table(n_req, V, length, 5)
    d_first, d_after = torch.tensor(first).cuda(), torch.tensor(after).cuda()

    def next_logits(t, tokens):
        z = d_first.repeat_interleave(B, 0) if t == 0 else d_after[t][tokens.clamp(min=0).long()]
        if t == 2:
            z[:B] = math.nan
        z[2 * B:, 2:] = -math.inf  # two tokens: two beams after the first
        return z

    stream = pr.StreamState(n_req * B, max_len)
    slots = torch.arange(n_req * B, dtype=torch.int32, device="cuda").view(n_req, B)
    out = bs.beam_search(next_logits, n_req, B, 1, 1.0, None, (), stream, slots)
    there = out["scores"] > -math.inf
    assert there[0].all() and there[2].tolist() == [True, True, False]
    score = stream.finish(slots.view(-1), 0.0)["score"].view(n_req, B)
    assert torch.equal(score.isnan(), ~there)
    out = bs.beam_search(next_logits, n_req, B, length, 1.0, None, (), stream, slots)
    there = out["scores"] > -math.inf
    assert not there[0].any() and there[1].all()
    verdict = stream.finish(slots.view(-1), 0.0)
    assert torch.equal(verdict["score"].view(n_req, B).isnan(), ~there)
    assert not verdict["ship"].view(n_req, B)[~there].any()
    stream.close()
