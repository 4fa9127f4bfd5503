"""Performance cases of the training operators: what post-training a small model has them do.

A case names one operator and its sizes:

- ``policy``:     the clipped policy loss with a KL term over logit rows, its
                  per-token values and its gradient in the logits;
- ``preference``: the preference loss over pairs of requests, its per-pair and
                  per-request values and its gradient in the logits;
- ``adamw``:      one AdamW step over many tensors, states in 32 or 8 bits.

Each has its plain form here (elementary torch operations in float32); with
``own`` true the framework's entry points run instead.
"""

import math

import numpy as np
import torch

own = False

DEV = "cuda"
CHUNK = 256 * 262144  # logits handled together while inputs or exact values are made
BLOCK = 256           # elements that share an exponent in 8-bit states
MASKED, CLIPPED = 16, 32
STEP0 = 100           # steps taken before the measured one
HYPER = dict(lr=3e-4, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, grad_scale=1.0)
SEED = 20             # of the stochastic rounding

# The parameter tensors of the verifier's transformer head: projection, two
# encoder layers (qkv, out, norm, feed-forward, norm), output.
HEAD = [64 * 4, 64] + 2 * [192 * 64, 192, 64 * 64, 64, 64, 64, 128 * 64, 128, 64 * 128, 64, 64, 64] + [64, 1]
# A small model: an output layer over 151,936 tokens at width 1,024 and four blocks (norms, q, k, v, o, gated feed-forward).
MODEL = [151936 * 1024] + 4 * [1024, 1024 * 1024, 256 * 1024, 256 * 1024, 1024 * 1024, 1024, 4096 * 1024, 4096 * 1024,
                               1024 * 4096] + [1024]


def listed():
    return [
        # The reference batch: 8 answers of 64 tokens, V = 32,000 float32.
        dict(name="policy_8x64_v32000_f32", op="policy", n_req=8, len_lo=64, len_hi=64, V=32000, dtype="f32", T=1.0,
             masked=0.0, kl=0.02),
        # The benchmark's batch: 64 ragged answers, V = 151,936 bfloat16, T = 0.7; some tokens do not count. The largest.
        dict(name="policy_64req_v151936_bf16", op="policy", n_req=64, len_lo=16, len_hi=512, V=151936, dtype="bf16",
             T=0.7, masked=0.1, kl=0.02),
        # One short answer on a vocabulary that is no multiple of a vector: latency counts. No reference model.
        dict(name="policy_1x17_v50257_bf16", op="policy", n_req=1, len_lo=17, len_hi=17, V=50257, dtype="bf16", T=1.0,
             masked=0.0, kl=0.0),
        # Float32 rows of 1 MB, half the tokens do not count (tool output inside the answers).
        dict(name="policy_16x128_v262144_f32", op="policy", n_req=16, len_lo=128, len_hi=128, V=262144, dtype="f32",
             T=1.0, masked=0.5, kl=0.05),
        # One pair of short answers.
        dict(name="preference_1pair_v32000_f32", op="preference", n_req=2, len_lo=1, len_hi=24, V=32000, dtype="f32",
             T=1.0, masked=0.0, smooth=0.0, ref=1, mean=0),
        # Eight pairs on an odd vocabulary; label smoothing.
        dict(name="preference_8pairs_v50257_bf16", op="preference", n_req=16, len_lo=1, len_hi=200, V=50257,
             dtype="bf16", T=1.0, masked=0.2, smooth=0.1, ref=1, mean=0),
        # The benchmark's batch as 32 pairs; prompts inside the rows do not count.
        dict(name="preference_32pairs_v151936_bf16", op="preference", n_req=64, len_lo=16, len_hi=512, V=151936,
             dtype="bf16", T=1.0, masked=0.1, smooth=0.0, ref=1, mean=0),
        # Mean log-probs with a margin and no reference model, float32.
        dict(name="preference_8pairs_v151936_f32", op="preference", n_req=16, len_lo=64, len_hi=256, V=151936,
             dtype="f32", T=1.0, masked=0.0, smooth=0.0, ref=0, mean=1),
        # The verifier's head: 28 small float32 tensors. Latency counts.
        dict(name="adamw_head_f32", op="adamw", kind="head", count=len(HEAD), most=0, param="f32", grad="f32", bits=32),
        # A small model in mixed precision: float32 weights with a bfloat16 copy, bfloat16 gradients.
        dict(name="adamw_model_f32_copy", op="adamw", kind="model", count=len(MODEL), most=0, param="f32+copy",
             grad="bf16", bits=32),
        # The same with 8-bit states.
        dict(name="adamw_model_8bit", op="adamw", kind="model", count=len(MODEL), most=0, param="f32+copy",
             grad="bf16", bits=8),
        # Many tensors of odd sizes in bfloat16 (adapters, norms, biases), 8-bit states.
        dict(name="adamw_300_odd_bf16_8bit", op="adamw", kind="odd", count=300, most=200000, param="bf16", grad="bf16",
             bits=8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("policy", "policy", "preference", "preference", "adamw"))
    if op == "adamw":
        count = _log_int(rng, 1, 400)
        return dict(op=op, kind="odd", count=count, most=_log_int(rng, 1000, 200_000_000 // count),
                    param=rng.choice(("f32", "f32+copy", "bf16")), grad=rng.choice(("f32", "bf16")),
                    bits=rng.choice((8, 32)))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    V = rng.choice((32000, 50257, 65536, 128003, 131072, 151936, 151936, 262144))
    rows = _log_int(rng, 4, 4.0e9 / (V * (2 if dtype == "bf16" else 4)))
    lo = _log_int(rng, 1, 128)
    hi = max(lo, min(_log_int(rng, lo, 512), rows // 2))
    lo = min(lo, hi)
    n_req = max(1, min(256, rows // hi))
    c = dict(op=op, V=V, dtype=dtype, T=rng.choice((0.5, 0.7, 1.0, 1.0)), len_lo=lo, len_hi=hi,
             masked=rng.choice((0.0, 0.1, 0.3, 0.6)))
    if op == "policy":
        return dict(c, n_req=n_req, kl=rng.choice((0.0, 0.02, 0.05)))
    mean = rng.randint(0, 1)
    return dict(c, n_req=2 * max(1, n_req // 2), smooth=rng.choice((0.0, 0.1)), ref=1 - mean, mean=mean)


# ---------------------------------------------------------------------------
# Sizes: part of the case, the same for every seed

def _lengths(case):
    rng = np.random.default_rng([case["n_req"], case["len_lo"], case["len_hi"]])
    return rng.integers(case["len_lo"], case["len_hi"] + 1, size=case["n_req"]).astype(np.int64)


def _active(case):
    """Which rows count: tokens left out at random, and every eighth request whole."""
    L = _lengths(case)
    rng = np.random.default_rng([int(L.sum()), int(case["masked"] * 1000)])
    on = rng.random(int(L.sum())) >= case["masked"]
    if case["masked"]:
        on &= np.repeat(np.arange(len(L)) % 8 != 5, L)
        on[0] = True
    return on


def _sizes(case):
    if case["kind"] == "head":
        return HEAD
    if case["kind"] == "model":
        return MODEL
    rng = np.random.default_rng([case["count"], case["most"]])
    return [int(v) for v in np.exp(rng.uniform(0.0, math.log(case["most"]), size=case["count"])).round()]


def work(case):
    if case["op"] == "adamw":
        n = sum(_sizes(case))
        blocks = sum(-(-k // BLOCK) for k in _sizes(case))
        p = {"f32": 8, "f32+copy": 10, "bf16": 4}[case["param"]]
        g = 4 if case["grad"] == "f32" else 2
        if case["bits"] == 32:
            return {"bytes": n * (p + g + 16), "flops": 14.0 * n}
        # codes and exponents in and out, and the states' values returned
        return {"bytes": n * (p + g + 4 + 4) + 4 * blocks, "flops": 30.0 * n}
    on = _active(case)
    item = 2 if case["dtype"] == "bf16" else 4
    n, a, V = len(on), int(on.sum()), case["V"]
    return {"bytes": (n + a) * V * item + n * 48, "flops": 10.0 * a * V}


# ---------------------------------------------------------------------------
# Inputs

def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 2654435761 % (1 << 62) + 1)
    return g


def _rows(case, g, looser=None):
    """Logits (a row's values at its own scale, one likely token each; a padded vocabulary in every eighth row), the
    tokens drawn from softmax(z / T) (at 2 T where `looser`) and their log-probs. Rows that do not count hold whatever
    was there."""
    on = torch.from_numpy(_active(case)).to(DEV)
    n, V, T = len(on), case["V"], case["T"]
    out = torch.empty(n, V, dtype=torch.bfloat16 if case["dtype"] == "bf16" else torch.float32, device=DEV)
    ids = torch.empty(n, dtype=torch.int32, device=DEV)
    logp = torch.empty(n, device=DEV)
    s = torch.empty(n, 1, device=DEV).uniform_(1.0, 4.0, generator=g)
    h = torch.empty(n, 1, device=DEV).uniform_(0.0, 15.0, generator=g)
    j = torch.randint(0, V - V // 16, (n, 1), generator=g, device=DEV)
    step = max(1, CHUNK // V)
    for a in range(0, n, step):
        b = min(n, a + step)
        z = torch.empty(b - a, V, device=DEV).normal_(generator=g).mul_(s[a:b])
        z.scatter_add_(1, j[a:b], h[a:b])
        z[(-a) % 8::8, V - V // 16:] = -math.inf
        out[a:b] = z
        z = out[a:b].float() / T
        lp = torch.log_softmax(z, dim=1)
        race = torch.empty_like(z).exponential_(generator=g).clamp_(min=1e-30)
        drawn = lp if looser is None else torch.where(looser[a:b, None], 0.5 * lp, lp)
        y = torch.argmax(drawn - race.log(), dim=1, keepdim=True)
        ids[a:b] = y[:, 0].to(torch.int32)
        logp[a:b] = lp.gather(1, y)[:, 0]
    out[~on & (torch.arange(n, device=DEV) % 3 == 0)] = math.nan
    return out, ids, logp, on


def _normal(n, g):
    return torch.empty(n, device=DEV).normal_(generator=g)


def _encode(x, rnd, expo_bits, floor):
    """Codes of 3 mantissa bits and `expo_bits` exponent bits of |x| [blocks, 256], and each block's exponent. rnd:
    20 random bits an element. floor: the least code of a value above zero."""
    bits = x.abs().view(torch.int32)
    top = (1 << expo_bits) - 1
    e = ((bits.amax(1, keepdim=True) + 0xFFFFF) >> 23).clamp(min=top + 1)
    k = ((bits + rnd) >> 20) - 8 * (e - top)
    k = torch.where(bits > 0, k.clamp(min=floor), 0)
    return k, e


def _decode(k, e, expo_bits):
    """Values of codes k (int32 [blocks, 256]) under block exponents e ([blocks, 1])."""
    top = (1 << expo_bits) - 1
    x = ((k + 8 * (e - top)) << 20).view(torch.float32)
    return torch.where(k > 0, x, 0.0)


def _key32(seed, step):
    """32 bits for a step's random numbers (the output function of SplitMix64)."""
    M = (1 << 64) - 1
    x = (seed + step * 0x9E3779B97F4A7C15) & M
    x = ((x ^ (x >> 30)) * 0xBF58476D1CE4E5B9) & M
    x = ((x ^ (x >> 27)) * 0x94D049BB133111EB) & M
    return ((x ^ (x >> 31)) >> 32) & 0xFFFFFFFF


def _mix(x):
    """32 random bits of each counter (int64 holding 32 bits)."""
    x = (x * 0x9E3779B9) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    return x ^ (x >> 13)


def _random_bits(tensor, first, seed, step):
    """32 bits for each element of the blocks: block b holds elements first[b].. of tensor[b]."""
    key = _mix((tensor + 1 + _key32(seed, step)) & 0xFFFFFFFF)
    return _mix((first[:, None] + torch.arange(BLOCK, device=DEV) + key[:, None]) & 0xFFFFFFFF)


def _split(flat, sizes, starts):
    return [flat[a:a + k] for k, a in zip(sizes, starts)]


def _prepare_adamw(case, g):
    sizes = _sizes(case)
    blocks = [-(-k // BLOCK) for k in sizes]
    starts = [BLOCK * int(v) for v in np.cumsum([0] + blocks[:-1])]
    total = BLOCK * sum(blocks)
    # Every tensor is a stretch of one buffer that starts at a multiple of 256 elements; zeros lie between.
    live = torch.zeros(total, dtype=torch.bool, device=DEV)
    for k, a in zip(sizes, starts):
        live[a:a + k] = True
    tensor = torch.from_numpy(np.repeat(np.arange(len(sizes)), blocks)).to(DEV)
    first = torch.from_numpy(np.concatenate([np.arange(b) for b in blocks]) * BLOCK).to(DEV)
    scale = torch.exp(_normal(sum(blocks), g))[:, None]  # gradients of a block at its own scale
    dead = torch.rand(sum(blocks), 1, generator=g, device=DEV) < 0.02  # rows that no token has used yet
    live &= (~dead).expand(-1, BLOCK).reshape(-1)
    st = {"case": case, "sizes": sizes, "starts": starts, "tensor": tensor, "first": first, "t": STEP0}

    def make(width, power=1):
        x = _normal(total, g).view(-1, BLOCK).mul_(scale).mul_(width)
        x = x if power == 1 else x.square_()
        return x.view(-1).mul_(live)

    grad = make(1e-3)
    st["grad"] = grad if case["grad"] == "f32" else grad.bfloat16()
    st["param"] = (_normal(total, g).mul_(0.02).mul_(live)).to(torch.bfloat16 if case["param"] == "bf16" else torch.float32)
    if case["param"] == "f32+copy":
        st["copy"] = st["param"].bfloat16()
    m = make(3e-4)
    v = make(8e-4, 2).add_(1e-7 * scale.square().expand(-1, BLOCK).reshape(-1)).mul_(live)
    if case["bits"] == 32:
        st["m"], st["v"] = m, v
    else:
        rnd = _random_bits(tensor, first, SEED, 0)
        m, v = m.view(-1, BLOCK), v.view(-1, BLOCK)
        k, e = _encode(m, (rnd & 0xFFFFF).int(), 4, 0)
        st["m"] = (k | torch.where(m < 0, 128, 0)).to(torch.uint8).view(-1)
        st["m_exp"] = e[:, 0].to(torch.uint8)
        k, e = _encode(v, (rnd >> 12).int(), 5, 1)
        st["v"] = k.to(torch.uint8).view(-1)
        st["v_exp"] = e[:, 0].to(torch.uint8)
        st["m_value"], st["v_value"] = (torch.zeros(total, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    if own:
        import paper_2608_28726_amd as pr
        part = {k: _split(st[k], sizes, starts) for k in ("param", "grad", "copy", "m", "v") if k in st}
        if case["bits"] == 8:
            at = [a // BLOCK for a in starts]
            part.update({k: _split(st[k], blocks, at) for k in ("m_exp", "v_exp")})
        states = [{k: part[k][i] for k in ("m", "v", "m_exp", "v_exp") if k in part} for i in range(len(sizes))]
        st["opt"] = pr.AdamW(part["param"], grads=part["grad"], copies=part.get("copy"), state_bits=case["bits"],
                             states=states, seed=SEED, steps=STEP0)
    return st


def _off_boundary(x, at):
    """x with no value within 1e-3 of `at`: a ratio that near the clip may fall on either side of it."""
    return torch.where((x - at).abs() < 1e-3, at + 2e-3, x)


def prepare(case, seed):
    g = _generator(seed)
    if case["op"] == "adamw":
        return _prepare_adamw(case, g)
    L = _lengths(case)
    req = torch.from_numpy(np.repeat(np.arange(len(L)), L)).to(DEV)
    # The rejected answers of a preference are less likely ones.
    logits, ids, logp, on = _rows(case, g, req % 2 == 1 if case["op"] == "preference" else None)
    n = len(on)
    st = {"case": case, "logits": logits, "ids": ids, "T": torch.full((n,), case["T"], device=DEV)}
    if case["op"] == "policy":
        delta = _off_boundary(_off_boundary(0.25 * _normal(n, g), math.log(0.8)), math.log(1.3))
        st["old"] = logp - delta
        st["ref"] = logp + 0.3 * _normal(n, g) if case["kl"] else None
        per_request = 0.5 + torch.rand(len(L), generator=g, device=DEV) * 2 - 0.75
        st["advantage"] = per_request[req] + 0.3 * _normal(n, g)
        st["weight"] = on.float() / int(_active(case).sum())
        return st
    off = np.zeros(len(L) + 1, dtype=np.int32)
    off[1:] = np.cumsum(L)
    st["offsets"] = torch.from_numpy(off).to(DEV)
    # Some steps into training: the chosen answers have become likelier than the reference has them.
    drift = torch.where(req % 2 == 0, 0.1, -0.1) * (0.5 + torch.rand(n, generator=g, device=DEV))
    st["ref"] = logp - drift - 0.05 * _normal(n, g) if case["ref"] else None
    st["weight"] = on.float()
    if case["mean"]:
        count = np.maximum(np.add.reduceat(_active(case).astype(np.float32), off[:-1]), 1.0).astype(np.float32)
        st["weight"] /= torch.from_numpy(count).to(DEV)[req]
    return st


# ---------------------------------------------------------------------------
# One pass

def _policy_options(case):
    return dict(clip_low=0.2, clip_high=0.3, kl_coef=case["kl"], grad_scale=1.0)


def _preference_options(case):
    return dict(beta=2.0 if case["mean"] else 0.1, label_smoothing=case["smooth"], margin=0.5 if case["mean"] else 0.0,
                grad_scale=1.0)


def run(st):
    case = st["case"]
    if not own:
        return {"policy": _plain_policy, "preference": _plain_preference, "adamw": _plain_adamw}[case["op"]](st, case)
    import paper_2608_28726_amd as pr
    if case["op"] == "policy":
        return pr.policy_loss(st["logits"], st["ids"], st["T"], st["weight"], st["advantage"], st["old"], st["ref"],
                              **_policy_options(case))
    if case["op"] == "preference":
        return pr.preference_loss(st["logits"], st["ids"], st["T"], st["weight"], st["offsets"], st["ref"],
                                  **_preference_options(case))
    st["opt"].step(**HYPER)
    if case["bits"] == 8:
        st["opt"].moments(out=(st["m_value"], st["v_value"]))
    return _adamw_outputs(st)


def _adamw_outputs(st):
    names = ("m", "v") if st["case"]["bits"] == 32 else ("m_value", "v_value")
    out = {"param": st["param"], "m": st[names[0]], "v": st[names[1]]}
    if "copy" in st:
        out["copy"] = st["copy"]
    return out


def _log_probs(st):
    """Per row: the token's log-prob, all probabilities, the one-hot token and whether the row counts."""
    on = st["weight"] != 0
    u = torch.where(on[:, None], st["logits"].float(), 0.0) / st["T"][:, None]
    u = u - u.amax(1, keepdim=True)
    e = torch.exp(u)
    S = e.sum(1, keepdim=True)
    y = st["ids"].long()[:, None]
    logp = torch.where(on, u.gather(1, y)[:, 0] - torch.log(S[:, 0]), 0.0)
    return logp, e / S, y, on


def _gradient(st, p, y, dl):
    """dl / T (onehot - p), in the logits' type."""
    c = (dl / st["T"])[:, None]
    return (-c * p).scatter_add_(1, y, c).to(st["logits"].dtype)


def _plain_policy(st, case):
    o = _policy_options(case)
    w, A = st["weight"], st["advantage"]
    logp, p, y, on = _log_probs(st)
    ratio = torch.exp(logp - st["old"])
    free, held = ratio * A, ratio.clamp(1 - o["clip_low"], 1 + o["clip_high"]) * A
    clipped = free > held
    d = st["ref"] - logp if st["ref"] is not None else torch.zeros_like(logp)
    rise = torch.expm1(d)
    kl = rise - d
    loss = torch.where(on, w * (o["kl_coef"] * kl - torch.minimum(free, held)), 0.0).sum().reshape(1)
    dl = torch.where(on, w * (torch.where(clipped, 0.0, -free) - o["kl_coef"] * rise), 0.0) * o["grad_scale"]
    return {"loss": loss, "logprob": logp, "ratio": torch.where(on, ratio, 0.0), "kl": torch.where(on, kl, 0.0),
            "flags": torch.where(on, torch.where(clipped, CLIPPED, 0), MASKED).int(),
            "grad": _gradient(st, p, y, dl)}


def _plain_preference(st, case):
    o = _preference_options(case)
    w, off = st["weight"], st["offsets"].long()
    logp, p, y, on = _log_probs(st)
    t = torch.where(on, w * (logp - st["ref"] if st["ref"] is not None else logp), 0.0)
    n_req = case["n_req"]
    req = torch.repeat_interleave(torch.arange(n_req, device=DEV), off[1:] - off[:-1], output_size=len(on))
    q = torch.zeros(n_req, device=DEV).index_add_(0, req, t)
    h = o["beta"] * (q[0::2] - q[1::2]) - o["margin"]
    s = o["label_smoothing"]
    tail = torch.log1p(torch.exp(-h.abs()))
    pair = (1 - s) * (tail + (-h).clamp(min=0)) + s * (tail + h.clamp(min=0))
    dh = (s / (1 + torch.exp(-h)) - (1 - s) / (1 + torch.exp(h))) / len(h)
    dq = torch.stack([dh, -dh], 1).reshape(-1) * o["beta"]
    dl = torch.where(on, w * dq[req], 0.0) * o["grad_scale"]
    return {"loss": pair.mean().reshape(1), "pair_loss": pair, "pair_logit": h, "seq_logratio": q, "logprob": logp,
            "flags": torch.where(on, 0, MASKED).int(), "grad": _gradient(st, p, y, dl)}


def _plain_adamw(st, case):
    st["t"] += 1
    o = HYPER
    g = (st["grad"].float() * o["grad_scale"]).view(-1, BLOCK)
    p = st["param"].float().view(-1, BLOCK)
    c1, c2 = 1 / (1 - o["beta1"] ** st["t"]), 1 / math.sqrt(1 - o["beta2"] ** st["t"])
    if case["bits"] == 8:
        mk = st["m"].view(-1, BLOCK).int()
        m = _decode(mk & 127, st["m_exp"].int()[:, None], 4) * torch.where(mk > 127, -1.0, 1.0)
        v = _decode(st["v"].view(-1, BLOCK).int(), st["v_exp"].int()[:, None], 5)
    else:
        m, v = st["m"].view(-1, BLOCK), st["v"].view(-1, BLOCK)
    m = m * o["beta1"] + g * (1 - o["beta1"])
    v = v * o["beta2"] + (g * g) * (1 - o["beta2"])
    p = p * (1 - o["lr"] * o["weight_decay"]) - (o["lr"] * c1) * m / (c2 * torch.sqrt(v) + o["eps"])
    if case["bits"] == 8 or case["param"] == "bf16":
        rnd = _random_bits(st["tensor"], st["first"], SEED, st["t"])
    if case["param"] == "bf16":
        up = ((p.view(torch.int32) + (rnd & 0xFFFF).int()) >> 16) << 16
        st["param"].copy_(up.view(torch.float32).view(-1))
    else:
        st["param"].copy_(p.view(-1))
        if "copy" in st:
            st["copy"].copy_(p.view(-1))
    if case["bits"] == 32:
        st["m"].copy_(m.view(-1))
        st["v"].copy_(v.view(-1))
        return _adamw_outputs(st)
    k, e = _encode(m, (rnd & 0xFFFFF).int(), 4, 0)
    st["m"].copy_((k | torch.where(m < 0, 128, 0)).view(-1))
    st["m_exp"].copy_(e[:, 0])
    st["m_value"].copy_((_decode(k, e, 4) * torch.where(m < 0, -1.0, 1.0)).view(-1))
    k, e = _encode(v, (rnd >> 12).int(), 5, 1)
    st["v"].copy_(k.view(-1))
    st["v_exp"].copy_(e[:, 0])
    st["v_value"].copy_(_decode(k, e, 5).view(-1))
    return _adamw_outputs(st)


# ---------------------------------------------------------------------------
# The same outputs in 64 bits, from the definitions

def _exact_log_probs(st):
    """log p_y of every row that counts, its normaliser and the row's largest scaled logit."""
    n, V = st["logits"].shape
    T = float(np.float32(st["case"]["T"]))
    on = st["weight"] != 0
    out = torch.zeros(n, dtype=torch.float64, device=DEV)
    lse = torch.zeros(n, dtype=torch.float64, device=DEV)
    step = max(1, CHUNK // 2 // V)
    for a in range(0, n, step):
        b = min(n, a + step)
        u = st["logits"][a:b].double() / T
        lse[a:b] = torch.logsumexp(u, 1)
        out[a:b] = u.gather(1, st["ids"][a:b].long()[:, None])[:, 0] - lse[a:b]
    return torch.where(on, out, 0.0), lse, on


def _exact_gradient(st, lse, on, dl):
    n, V = st["logits"].shape
    T = float(np.float32(st["case"]["T"]))
    out = torch.zeros(n, V, dtype=torch.float64, device=DEV)
    step = max(1, CHUNK // 2 // V)
    for a in range(0, n, step):
        b = min(n, a + step)
        rows = on[a:b].nonzero()[:, 0]
        z = st["logits"][a:b][rows].double() / T
        d = -torch.exp(z - lse[a:b][rows][:, None])
        d[torch.arange(len(rows), device=DEV), st["ids"][a:b][rows].long()] += 1.0
        out[a:b][rows] = d * (dl[a:b][rows] / T)[:, None]
    return out


def _exact_policy(st, case):
    o = _policy_options(case)
    logp, lse, on = _exact_log_probs(st)
    w, A = st["weight"].double(), st["advantage"].double()
    x = torch.exp(logp - st["old"].double())
    lo, hi = 1.0 - o["clip_low"], 1.0 + o["clip_high"]
    clipped = ((A > 0) & (x > hi)) | ((A < 0) & (x < lo))
    gain = torch.where(clipped, torch.where(A > 0, hi, lo) * A, x * A)
    ref = st["ref"].double() if st["ref"] is not None else logp
    kl = torch.expm1(ref - logp) - (ref - logp)
    loss = torch.where(on, w * (o["kl_coef"] * kl - gain), 0.0)
    dl = torch.where(on, w * (torch.where(clipped, 0.0, -x * A) - o["kl_coef"] * torch.expm1(ref - logp)), 0.0)
    return {"loss": loss.sum().reshape(1), "logprob": logp, "ratio": torch.where(on, x, 0.0),
            "kl": torch.where(on, kl, 0.0), "flags": torch.where(on, torch.where(clipped, CLIPPED, 0), MASKED).int(),
            "grad": _exact_gradient(st, lse, on, dl)}


def _exact_preference(st, case):
    o = _preference_options(case)
    logp, lse, on = _exact_log_probs(st)
    off = st["offsets"].tolist()
    term = st["weight"].double() * (logp - (st["ref"].double() if st["ref"] is not None else 0.0))
    term = torch.where(on, term, 0.0)
    q = torch.stack([term[off[i]:off[i + 1]].sum() for i in range(case["n_req"])])
    h = o["beta"] * (q[0::2] - q[1::2]) - o["margin"]
    s = o["label_smoothing"]
    logsig = torch.nn.functional.logsigmoid
    pair = -(1 - s) * logsig(h) - s * logsig(-h)
    dh = (torch.sigmoid(h) - (1 - s)) / len(h)
    dl = torch.zeros_like(logp)
    for i in range(case["n_req"]):
        a, b = off[i], off[i + 1]
        dl[a:b] = st["weight"][a:b].double() * o["beta"] * dh[i // 2] * (1 if i % 2 == 0 else -1)
    return {"loss": pair.mean().reshape(1), "pair_loss": pair, "pair_logit": h, "seq_logratio": q, "logprob": logp,
            "flags": torch.where(on, 0, MASKED).int(), "grad": _exact_gradient(st, lse, on, dl)}


def _exact_values(x, rnd, expo_bits, floor):
    """What 64-bit values x [blocks, 256] become in 8 bits. A positive value at 8 (exponent + 127 + fraction) on the
    scale of codes is rounded up with the probability of its fraction there."""
    top = (1 << expo_bits) - 1
    mant, ex = torch.frexp(x.abs())
    place = torch.where(x != 0, 8.0 * (ex + 125 + 2 * mant), 0.0).clamp(min=0.0)
    e = torch.floor((place.amax(1, keepdim=True) + (1 - 2.0 ** -20)) / 8).clamp(min=top + 1)
    code = torch.floor(place + rnd * 2.0 ** -20) - 8 * (e - top)
    code = torch.where(x != 0, code.clamp(min=floor), 0.0)
    whole = torch.floor((code + 8 * (e - top)) / 8)
    value = (1 + (code + 8 * (e - top)) / 8 - whole) * torch.exp2(whole - 127)
    return torch.where(code > 0, value, 0.0) * torch.sign(x)


def _exact_adamw(st, case):
    o, t = HYPER, STEP0 + 1
    g = st["grad"].double().view(-1, BLOCK) * o["grad_scale"]
    p = st["param"].double().view(-1, BLOCK)
    if case["bits"] == 8:
        mk, vk = (st[k].view(-1, BLOCK).double() for k in ("m", "v"))
        me, ve = (st[k].double()[:, None] for k in ("m_exp", "v_exp"))

        def value(code, e, top):
            at = code + 8 * (e - top)
            return torch.where(code > 0, (1 + at / 8 - torch.floor(at / 8)) * torch.exp2(torch.floor(at / 8) - 127), 0.0)

        m = value(mk % 128, me, 15) * torch.where(mk >= 128, -1.0, 1.0)
        v = value(vk, ve, 31)
    else:
        m, v = st["m"].double().view(-1, BLOCK), st["v"].double().view(-1, BLOCK)
    m = o["beta1"] * m + (1 - o["beta1"]) * g
    v = o["beta2"] * v + (1 - o["beta2"]) * g * g
    mh, vh = m / (1 - o["beta1"] ** t), v / (1 - o["beta2"] ** t)
    p = p - o["lr"] * o["weight_decay"] * p - o["lr"] * mh / (vh.sqrt() + o["eps"])
    if case["bits"] == 8:
        rnd = _random_bits(st["tensor"], st["first"], SEED, t)
        m = _exact_values(m, rnd & 0xFFFFF, 4, 0)
        v = _exact_values(v, rnd >> 12, 5, 1)
    out = {"param": p.view(-1), "m": m.view(-1), "v": v.view(-1)}
    if "copy" in st:
        out["copy"] = p.view(-1)
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return {"policy": _exact_policy, "preference": _exact_preference, "adamw": _exact_adamw}[case["op"]](st, case)
