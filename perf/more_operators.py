"""Performance cases of beam search and distillation: what a teacher's decoding and a student's training on it have them do.

A case names one operator and its sizes:

- ``top``:     the k largest logits of each row with their log-probs (what is kept of a teacher's answer);
- ``distill``: the loss of a student's rows against a teacher's top log-probs, its per-token values and its gradient
               in the logits;
- ``select``:  a step of beam search: the k best continuations of each request's beams over the vocabulary;
- ``reorder``: the beams' states put into the order of the beams that were chosen, in place.

Each has its plain form here (elementary torch operations); with ``own`` true the framework's entry points run instead.
"""

import math

import numpy as np
import torch

own = False

DEV = "cuda"
CHUNK = 256 * 262144  # logits handled together while inputs, plain selections or exact values are made
MASKED = 16
NONE = -1             # an id that stands for no token
APART = 2e-5          # least distance of two beams' candidates next to each other


def listed():
    return [
        # The reference batch, 8 answers of 64 tokens at V = 32,000 float32, with the paper's K.
        dict(name="top20_8x64_v32000_f32", op="top", n_req=8, len_lo=64, len_hi=64, V=32000, dtype="f32", T=1.0, k=20),
        # The benchmark's batch, 64 ragged answers at V = 151,936 bfloat16: a teacher's 64 best of each token.
        dict(name="top64_64req_v151936_bf16", op="top", n_req=64, len_lo=16, len_hi=512, V=151936, dtype="bf16", T=0.7,
             k=64),
        # One short answer, many of its logits, a vocabulary that is no multiple of a vector.
        dict(name="top256_1x17_v50257_bf16", op="top", n_req=1, len_lo=17, len_hi=17, V=50257, dtype="bf16", T=1.0,
             k=256),
        # The reference batch as a student's.
        dict(name="distill20_8x64_v32000_f32", op="distill", n_req=8, len_lo=64, len_hi=64, V=32000, dtype="f32", T=1.0,
             k=20, masked=0.0, tail="rest"),
        # The benchmark's batch as a student's; some tokens do not count. The largest.
        dict(name="distill64_64req_v151936_bf16", op="distill", n_req=64, len_lo=16, len_hi=512, V=151936, dtype="bf16",
             T=0.7, k=64, masked=0.1, tail="rest"),
        # One short answer: latency counts. What the teacher's tokens leave over is left out.
        dict(name="distill256_1x17_v50257_bf16", op="distill", n_req=1, len_lo=17, len_hi=17, V=50257, dtype="bf16",
             T=1.0, k=256, masked=0.0, tail="drop"),
        # Float32 rows of 1 MB, half the tokens do not count; the teacher's probabilities add to 1.
        dict(name="distill128_16x128_v262144_f32", op="distill", n_req=16, len_lo=128, len_hi=128, V=262144,
             dtype="f32", T=1.0, k=128, masked=0.5, tail="renorm"),
        # One request of four beams: latency counts.
        dict(name="select_1x4_v32000_f32", op="select", n_req=1, beams=4, k=4, V=32000, dtype="f32", T=1.0, done=0.0),
        # The decode stream's 256 rows as 64 requests of four beams; twice as many candidates as beams.
        dict(name="select_64x4_v151936_bf16", op="select", n_req=64, beams=4, k=8, V=151936, dtype="bf16", T=1.0,
             done=0.0),
        # Wide beams over float32 rows of 1 MB, some of them done.
        dict(name="select_32x16_v262144_f32", op="select", n_req=32, beams=16, k=16, V=262144, dtype="f32", T=0.8,
             done=0.2),
        # One request of four beams: its tokens so far and a recurrent state of 64 floats.
        dict(name="reorder_1x4_tokens", op="reorder", n_req=1, beams=4, layers=0, length=512, width=64, odd=0),
        # 64 requests of four beams: the keys and values of four blocks, 512 tokens of 256 bfloat16 each, and the tokens.
        dict(name="reorder_64x4_cache", op="reorder", n_req=64, beams=4, layers=4, length=512, width=256, odd=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("top", "distill", "distill", "select", "select", "reorder"))
    if op == "reorder":
        beams = rng.randint(2, 32)
        n_req = _log_int(rng, 1, 512 // beams)
        width, odd = rng.choice(((64, 0), (96, 0), (256, 0), (256, 0), (130, 1), (33, 1)))
        layers = rng.randint(0, 6)
        most = 600_000_000 // (n_req * beams * width * 2 * (2 * layers + 1))
        return dict(op=op, n_req=n_req, beams=beams, layers=layers, length=_log_int(rng, 1, max(1, min(4096, most))),
                    width=width, odd=odd)
    dtype = rng.choice(("bf16", "bf16", "f32"))
    V = rng.choice((32000, 50257, 65536, 128003, 131072, 151936, 151936, 262144))
    item = 2 if dtype == "bf16" else 4
    c = dict(op=op, V=V, dtype=dtype, T=rng.choice((0.5, 0.7, 1.0, 1.0)))
    if op == "select":
        beams = _log_int(rng, 1, 64)
        n_req = _log_int(rng, 1, max(1, int(0.54e9 / (beams * V * item))))
        k = rng.choice((beams, beams, 2 * beams, _log_int(rng, 1, 128)))
        return dict(c, n_req=n_req, beams=beams, k=k, done=rng.choice((0.0, 0.2, 0.5)) if k >= beams else 0.0)
    rows = _log_int(rng, 4, 4.0e9 / (V * item))
    lo = _log_int(rng, 1, 128)
    hi = max(lo, min(_log_int(rng, lo, 512), rows // 2))
    lo = min(lo, hi)
    c = dict(c, n_req=max(1, min(256, rows // hi)), len_lo=lo, len_hi=hi, k=_log_int(rng, 1, 256))
    if op == "top":
        return c
    return dict(c, masked=rng.choice((0.0, 0.1, 0.3, 0.6)), tail=rng.choice(("rest", "rest", "drop", "renorm")))


# ---------------------------------------------------------------------------
# Sizes: part of the case, the same for every seed

def _n_rows(case):
    if case["op"] in ("select", "reorder"):
        return case["n_req"] * case["beams"]
    rng = np.random.default_rng([case["n_req"], case["len_lo"], case["len_hi"]])
    return int(rng.integers(case["len_lo"], case["len_hi"] + 1, size=case["n_req"]).sum())


def _on(case):
    """Which rows take part."""
    n = _n_rows(case)
    share = case.get("masked", case.get("done", 0.0))
    on = np.random.default_rng([n, int(share * 1000)]).random(n) >= share
    on[0] = True
    return on


def _parents(case):
    """Who each beam follows: the better beams have more children."""
    B = case["beams"]
    rng = np.random.default_rng([case["n_req"], B, 7])
    return np.minimum((rng.random((case["n_req"], B)) ** 1.5 * B).astype(np.int32), B - 1)


def _states(case):
    """The shapes and types of a beam's states."""
    out = [((case["length"],), torch.int32), ((case["width"],), torch.float32)]
    return out + [((case["length"], case["width"]), torch.bfloat16)] * (2 * case["layers"])


def work(case):
    if case["op"] == "reorder":
        moved = int((_parents(case) != np.arange(case["beams"])[None]).sum())
        row = sum(math.prod(s) * (2 if t == torch.bfloat16 else 4) for s, t in _states(case))
        return {"bytes": 2 * moved * row + 4 * _n_rows(case), "flops": 0.0}
    item = 2 if case["dtype"] == "bf16" else 4
    on = _on(case)
    n, a, V, k = len(on), int(on.sum()), case["V"], case["k"]
    if case["op"] == "top":
        return {"bytes": n * (V * item + 8 * k + 12), "flops": 5.0 * n * V}
    if case["op"] == "select":
        return {"bytes": a * V * item + n * 12 + case["n_req"] * k * 16, "flops": 5.0 * a * V}
    return {"bytes": (n + a) * V * item + a * k * 8 + n * 20, "flops": 9.0 * a * V}


# ---------------------------------------------------------------------------
# Inputs

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 2654435761 % (1 << 62) + 1)
    return g


def _normal(shape, g):
    return torch.empty(shape, device=DEV).normal_(generator=g)


def _chunks(n, V):
    step = max(1, CHUNK // V)
    return [(a, min(n, a + step)) for a in range(0, n, step)]


def _logits(case, n, g):
    """Logits: a row's values at its own scale, one likely token each, a padded vocabulary in every eighth row."""
    V = case["V"]
    out = torch.empty(n, V, dtype=torch.bfloat16 if case["dtype"] == "bf16" else torch.float32, device=DEV)
    s = torch.empty(n, 1, device=DEV).uniform_(1.0, 4.0, generator=g)
    h = torch.empty(n, 1, device=DEV).uniform_(0.0, 15.0, generator=g)
    j = torch.randint(0, V - V // 16, (n, 1), generator=g, device=DEV)
    for a, b in _chunks(n, V):
        z = _normal((b - a, V), g).mul_(s[a:b])
        z.scatter_add_(1, j[a:b], h[a:b])
        z[(-a) % 8::8, V - V // 16:] = -math.inf
        out[a:b] = z
    return out


def _best_exact(logits, k, T):
    """The k largest logits of each row (float64, fewer than k of them are followed by -inf) and its log sum of exps."""
    n, V = logits.shape
    top = torch.full((n, k), -math.inf, dtype=torch.float64, device=DEV)
    lse = torch.empty(n, dtype=torch.float64, device=DEV)
    for a, b in _chunks(n, 2 * V):
        z = logits[a:b].double()
        top[a:b, :min(k, V)] = torch.topk(z, min(k, V), dim=1).values
        lse[a:b] = torch.logsumexp(z / T, 1)
    return top, lse


def _prepare_distill(case, g):
    n, V, k = _n_rows(case), case["V"], case["k"]
    logits = _logits(case, n, g)
    on = torch.from_numpy(_on(case)).to(DEV)
    ids = torch.empty(n, k, dtype=torch.int32, device=DEV)
    logq = torch.empty(n, k, device=DEV)
    width = torch.empty(n, 1, device=DEV).uniform_(0.1, 1.5, generator=g)
    for a, b in _chunks(n, V):  # the teacher's logits are the student's, sharpened and disturbed
        z = (logits[a:b].float() * (1.1 / case["T"])).add_(_normal((b - a, V), g).mul_(width[a:b]))
        top = torch.topk(z, k, dim=1)
        ids[a:b] = top.indices.to(torch.int32)
        logq[a:b] = top.values - torch.logsumexp(z, 1, keepdim=True)
    logq.clamp_(max=0.0)
    short = torch.arange(n, device=DEV) % 16 == 3  # rows of which fewer tokens were kept
    ids[short, k // 2:] = NONE
    logq[short, k // 2:] = -math.inf
    logits[~on & (torch.arange(n, device=DEV) % 3 == 0)] = math.nan
    return {"case": case, "logits": logits, "ids": ids, "logq": logq, "T": torch.full((n,), case["T"], device=DEV),
            "weight": on.float() / int(_on(case).sum())}


def _prepare_select(case, g):
    n_req, B, k = case["n_req"], case["beams"], case["k"]
    n = n_req * B
    logits = _logits(case, n, g)
    done = torch.from_numpy(~_on(case)).to(DEV).view(n_req, B)
    top, lse = _best_exact(logits, min(k + 1, case["V"]), float(np.float32(case["T"])))
    best = (top / float(np.float32(case["T"])) - lse[:, None]).view(n_req, B, -1)
    best = torch.where(done[..., None], -math.inf, best)
    best[..., 0] = torch.where(done, 0.0, best[..., 0])
    beam = torch.arange(B, device=DEV)[None, :, None].expand(best.shape).reshape(n_req, -1)
    scores = torch.zeros(n_req, B, device=DEV)
    again = torch.arange(n_req, device=DEV)
    for _ in range(100):  # running sums of log-probs; two beams' candidates do not come out next to equal
        scores[again] = _normal((len(again), B), g).mul_(2.0).sub_(20.0 + 5.0 * torch.rand((len(again), 1), generator=g,
                                                                                          device=DEV))
        s, at = (best[again] + scores[again].double()[..., None]).flatten(1).sort(1, descending=True)
        who = beam[again].gather(1, at)
        near = ((s[:, :-1] - s[:, 1:] < APART) & (who[:, :-1] != who[:, 1:]))[:, :k].any(1)
        again = again[near]
        if len(again) == 0:
            break
    return {"case": case, "logits": logits, "scores": scores, "done": done if case["done"] else None,
            "T": torch.full((n,), case["T"], device=DEV)}


def _prepare_reorder(case, g):
    n = _n_rows(case)
    states = []
    for shape, dtype in _states(case):
        # Rows of odd bytes from row to row where the case says so.
        row = math.prod(shape)
        buf = torch.empty(n * (row + case["odd"]), device=DEV, dtype=dtype)
        for a in range(0, buf.numel(), CHUNK):
            part = buf[a:a + CHUNK]
            if dtype == torch.int32:
                part.random_(0, 32000, generator=g)
            else:
                part.normal_(generator=g)
        states.append(buf.view(n, row + case["odd"])[:, :row])
    return {"case": case, "states": states, "parent": torch.from_numpy(_parents(case)).to(DEV)}


def prepare(case, seed):
    g = _generator(seed)
    if case["op"] == "top":
        n = _n_rows(case)
        return {"case": case, "logits": _logits(case, n, g), "T": torch.full((n,), case["T"], device=DEV)}
    return {"distill": _prepare_distill, "select": _prepare_select, "reorder": _prepare_reorder}[case["op"]](case, g)


# ---------------------------------------------------------------------------
# One pass

def run(st):
    case = st["case"]
    if not own:
        return {"top": _plain_top, "distill": _plain_distill, "select": _plain_select, "reorder": _plain_reorder}[
            case["op"]](st, case)
    import paper_2608_28726_amd as pr
    if case["op"] == "top":
        return pr.top_logits(st["logits"], case["k"], st["T"])
    if case["op"] == "distill":
        return pr.distill_loss(st["logits"], st["ids"], st["logq"], st["T"], st["weight"], tail=case["tail"])
    if case["op"] == "select":
        return pr.beam_select(st["logits"], st["scores"], st["T"], k=case["k"], done=st["done"], done_token=0)
    pr.beam_reorder(st["states"], st["parent"])
    return st["states"]


def _in_order(z, k):
    """The tokens of each row's k largest logits, larger ones first and equal ones by index, and those logits."""
    V = z.shape[1]
    bits = z.float().add(0.0).view(torch.int32).long()
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) * (1 << 32) + (V - 1 - torch.arange(V, device=DEV))
    ids = V - 1 - (torch.topk(key, min(k, V), dim=1).values & 0xFFFFFFFF)
    return ids, z.gather(1, ids).float()


def _row_best(logits, T, k):
    """Per row the first k tokens of its order, their log-probs and the log sum of exps (float32). Tokens of probability 0
    are none."""
    n, V = logits.shape
    ids = torch.full((n, k), NONE, dtype=torch.int32, device=DEV)
    logp = torch.full((n, k), -math.inf, device=DEV)
    lse = torch.empty(n, device=DEV)
    kk = min(k, V)
    for a, b in _chunks(n, 4 * V):
        z = logits[a:b]
        at, best = _in_order(z, kk)
        u = z.float() / T[a:b, None]
        top = u.amax(1, keepdim=True)
        over = torch.log(torch.exp(u - top).sum(1, keepdim=True))
        lse[a:b] = (top + over)[:, 0]
        logp[a:b, :kk] = (best / T[a:b, None] - top) - over
        ids[a:b, :kk] = torch.where(best > -math.inf, at, NONE).to(torch.int32)
    return ids, logp, lse


def _plain_top(st, case):
    ids, logp, lse = _row_best(st["logits"], st["T"], case["k"])
    return {"ids": ids, "logprob": logp, "lse": lse, "flags": torch.zeros(len(ids), dtype=torch.int32, device=DEV)}


def _plain_distill(st, case):
    on, w = st["weight"] != 0, st["weight"]
    kept = st["logq"] > -math.inf
    y = torch.where(kept, st["ids"], 0).long()
    q = torch.where(kept, torch.exp(st["logq"].double()), 0.0)
    Q = q.sum(1, keepdim=True)
    if case["tail"] == "renorm":
        some = kept.any(1, keepdim=True)
        logq = torch.where(kept, st["logq"] - torch.where(some, torch.log(Q), 0.0).float(), 0.0)
        q, Q = torch.where(some, q / Q, 0.0), some.double()
    else:
        logq = torch.where(kept, st["logq"], 0.0)
    left = (1 - Q).clamp(min=0).float()  # what the teacher's tokens leave over
    q, Q = q.float(), Q.float()
    u = torch.where(on[:, None], st["logits"].float(), 0.0) / st["T"][:, None]
    u = u - u.amax(1, keepdim=True)
    e = torch.exp(u)
    logS = torch.log(e.sum(1, keepdim=True))
    logp = u.gather(1, y) - logS
    loss = torch.where(kept, q * (logq - logp), 0.0).sum(1)
    P = torch.where(kept, torch.exp(logp), 0.0).sum(1, keepdim=True)
    # Which tokens are the teacher's, with their probabilities there
    target = torch.zeros_like(e).scatter_add_(1, y, q)
    mine = torch.zeros_like(e, dtype=torch.int8).scatter_add_(1, y, kept.to(torch.int8)) > 0
    p = e / torch.exp(logS)
    if case["tail"] == "rest":
        other = torch.where(mine, 0.0, e).sum(1, keepdim=True) / torch.exp(logS)
        has = (other > 0) & (left > 0)
        ratio = torch.where(has, left / other, 0.0)
        loss = loss + torch.where(has, left * torch.log(ratio), 0.0)[:, 0]
        du = torch.where(mine, (Q + torch.where(has, left, 0.0)) * p - target, (Q - ratio * P) * p)
    else:
        du = Q * p - target
    grad = du * torch.where(on, w / st["T"], 0.0)[:, None]
    loss = torch.where(on, loss, 0.0)
    return {"loss": (w * loss).sum().reshape(1), "token_loss": loss, "mass": torch.where(on, P[:, 0], 0.0),
            "flags": torch.where(on, 0, MASKED).int(), "grad": grad.to(st["logits"].dtype)}


def _plain_select(st, case):
    n_req, B, k = case["n_req"], case["beams"], case["k"]
    logits, T = st["logits"], st["T"].double()
    done = st["done"] if st["done"] is not None else torch.zeros(n_req, B, dtype=torch.bool, device=DEV)
    V = logits.shape[1]
    kk = min(k, V)
    ids = torch.empty(n_req * B, kk, dtype=torch.int32, device=DEV)
    logp = torch.empty(n_req * B, kk, dtype=torch.float64, device=DEV)
    for a, b in _chunks(n_req * B, 4 * V):  # in 64 bits: which candidate comes first hangs on them
        at, best = _in_order(logits[a:b], kk)
        u = logits[a:b].double() / T[a:b, None]
        top = u.amax(1, keepdim=True)
        logp[a:b] = best.double() / T[a:b, None] - top - torch.log(torch.exp(u - top).sum(1, keepdim=True))
        ids[a:b] = at
    first = torch.arange(kk, device=DEV) == 0
    logp = torch.where(done.view(-1, 1), torch.where(first, 0.0, -math.inf), logp)
    ids = torch.where(done.view(-1, 1), 0, ids).view(n_req, -1)
    s = (st["scores"].double()[..., None] + logp.view(n_req, B, kk)).view(n_req, -1)
    s, at = torch.sort(s, dim=1, descending=True, stable=True)
    s, at = s[:, :k], at[:, :k]
    out = {"scores": torch.full((n_req, k), -math.inf, device=DEV),
           "parent": torch.full((n_req, k), NONE, dtype=torch.int32, device=DEV),
           "token": torch.full((n_req, k), NONE, dtype=torch.int32, device=DEV),
           "logprob": torch.full((n_req, k), -math.inf, device=DEV)}
    found, m = s > -math.inf, s.shape[1]
    out["scores"][:, :m] = s.float()
    out["parent"][:, :m] = torch.where(found, at // kk, NONE).int()
    out["token"][:, :m] = torch.where(found, ids.gather(1, at), NONE)
    out["logprob"][:, :m] = logp.view(n_req, -1).gather(1, at).float()
    out["flags"] = torch.where(done, MASKED, 0).int().view(-1)
    return out


def _plain_reorder(st, case):
    rows = (torch.arange(case["n_req"], device=DEV)[:, None] * case["beams"] + st["parent"]).view(-1)
    for x in st["states"]:
        x.copy_(x[rows])
    return st["states"]


# ---------------------------------------------------------------------------
# The same outputs in 64 bits, from the definitions

def _exact_rows(logits, k, T):
    """The first k tokens of each row's order, their log-probs, the log sum of exps."""
    n, V = logits.shape
    kk = min(k, V)
    ids = torch.full((n, k), NONE, dtype=torch.int32, device=DEV)
    logp = torch.full((n, k), -math.inf, dtype=torch.float64, device=DEV)
    lse = torch.empty(n, dtype=torch.float64, device=DEV)
    for a, b in _chunks(n, 4 * V):
        z = logits[a:b].double()
        lse[a:b] = torch.logsumexp(z / T, 1)
        # Everything from the kk-th largest value on, by row and index, is sorted.
        floor = torch.topk(z, kk, dim=1).values[:, -1:]
        row, col = ((z >= floor) & (z > -math.inf)).nonzero(as_tuple=True)
        count = torch.bincount(row, minlength=b - a)
        place = torch.arange(len(row), device=DEV) - (torch.cumsum(count, 0) - count)[row]
        most = max(kk, int(count.amax()))
        v = torch.full((b - a, most), -math.inf, dtype=torch.float64, device=DEV)
        where = torch.full((b - a, most), NONE, dtype=torch.int64, device=DEV)
        v[row, place], where[row, place] = z[row, col], col
        v, at = torch.sort(v, dim=1, descending=True, stable=True)
        ids[a:b, :kk] = where.gather(1, at)[:, :kk].int()
        logp[a:b, :kk] = v[:, :kk] / T - lse[a:b, None]
    return ids, logp, lse


def _exact_distill(st, case):
    n, V = st["logits"].shape
    T = float(np.float32(case["T"]))
    grad = torch.zeros(n, V, dtype=torch.float64, device=DEV)
    token = torch.zeros(n, dtype=torch.float64, device=DEV)
    mass = torch.zeros(n, dtype=torch.float64, device=DEV)
    on = st["weight"] != 0
    for a, b in _chunks(n, 8 * V):
        rows = a + on[a:b].nonzero()[:, 0]
        logq = st["logq"][rows].double()
        kept = logq > -math.inf
        q = torch.exp(logq)
        some = kept.any(1).double()
        if case["tail"] == "renorm":
            logq = logq - torch.logsumexp(torch.where(kept, logq, -1e300), 1, keepdim=True)
            q = torch.where(kept, torch.exp(logq), 0.0)
        y = st["ids"][rows].long().clamp(min=0)
        logp = torch.log_softmax(st["logits"][rows].double() / T, 1)
        p = torch.exp(logp)
        entry = torch.arange(len(rows), device=DEV)[:, None].expand(y.shape)
        mine = torch.zeros_like(p)
        mine[entry[kept], y[kept]] = 1.0
        target = torch.zeros_like(p)
        target[entry[kept], y[kept]] = q[kept]
        at = logp.gather(1, y)
        token[rows] = torch.where(kept, q * (logq - at), 0.0).sum(1)
        Q, P = q.sum(1), (p * mine).sum(1)
        if case["tail"] == "renorm":
            Q = some
        over = torch.zeros_like(Q)
        outside = Q
        if case["tail"] == "rest":
            r = (p * (1 - mine)).sum(1)
            over = torch.where(r > 0, (1 - Q).clamp(min=0), 0.0)
            log_r = torch.logsumexp(torch.where(mine > 0, -math.inf, logp), 1)
            token[rows] += torch.where(over > 0, over * (torch.log(over) - log_r), 0.0)
            outside = Q - torch.where(over > 0, over * P / r, 0.0)
        du = torch.where(mine > 0, (Q + over)[:, None] * p - target, outside[:, None] * p)
        grad[rows] = du * (st["weight"][rows].double() / T)[:, None]
        mass[rows] = P
    return {"loss": (st["weight"].double() * token).sum().reshape(1), "token_loss": token, "mass": mass,
            "flags": torch.where(on, 0, MASKED).int(), "grad": grad}


def _exact_select(st, case):
    n_req, B, k = case["n_req"], case["beams"], case["k"]
    ids, logp, _ = _exact_rows(st["logits"], k, float(np.float32(case["T"])))
    ids, logp = ids.view(n_req, B, k).cpu().numpy(), logp.view(n_req, B, k).cpu().numpy()
    scores = st["scores"].double().cpu().numpy()
    done = st["done"].cpu().numpy() if st["done"] is not None else np.zeros((n_req, B), dtype=bool)
    out = {"scores": np.full((n_req, k), -np.inf), "parent": np.full((n_req, k), NONE, np.int32),
           "token": np.full((n_req, k), NONE, np.int32), "logprob": np.full((n_req, k), -np.inf)}
    for i in range(n_req):
        cand = []
        for b in range(B):
            if done[i, b]:
                cand.append((-scores[i, b], b, 0, 0, 0.0))
            else:
                cand += [(-(scores[i, b] + logp[i, b, j]), b, j, int(ids[i, b, j]), logp[i, b, j]) for j in range(k)
                         if ids[i, b, j] >= 0]
        for j, (s, b, _, token, lp) in enumerate(sorted(cand)[:k]):
            out["scores"][i, j], out["parent"][i, j], out["token"][i, j], out["logprob"][i, j] = -s, b, token, lp
    out = {name: torch.from_numpy(x).to(DEV) for name, x in out.items()}
    out["flags"] = torch.from_numpy(np.where(done, MASKED, 0).astype(np.int32)).to(DEV).view(-1)
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "top":
        ids, logp, lse = _exact_rows(st["logits"], case["k"], float(np.float32(case["T"])))
        return {"ids": ids, "logprob": logp, "lse": lse, "flags": torch.zeros(len(ids), dtype=torch.int32, device=DEV)}
    if case["op"] == "distill":
        return _exact_distill(st, case)
    if case["op"] == "select":
        return _exact_select(st, case)
    parent = st["parent"].long().cpu().tolist()
    out = []
    for x in st["states"]:
        rows = [x[i * case["beams"] + p] for i, row in enumerate(parent) for p in row]
        out.append(torch.stack(rows).double() if x.is_floating_point() else torch.stack(rows))
    return out
