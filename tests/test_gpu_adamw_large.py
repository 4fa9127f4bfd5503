"""AdamW steps over more than the last-level cache holds, which go past the caches: float32 parameters with copies and
bfloat16 ones, both kinds of states and gradients, odd tensors that start anywhere beside one that is large.

Tolerances as in test_gpu_adamw: states to the bit, parameters by check_param's bound.
"""

import numpy as np
import pytest
import torch

import paper_2608_28726_amd as pr
from oracle import adamw as oadam
from tests.gpu_common import require_gpu
from tests.test_gpu_adamw import HYPER, SIZES, U, check_param, f32_moments, host

pytestmark = pytest.mark.gpu

SEED, STEPS = 11, 3


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def make(n, dtype, g, scale, offset):
    t = torch.empty(n + offset + 3, device="cuda").normal_(generator=g).mul_(scale).to(dtype)
    return t[offset:offset + n]


def random_bits(n, tensor, step):
    """The documented random bits of a tensor's elements, on the device."""
    first = int(oadam.random_bits(1, tensor, SEED, step)[0])  # element 0's, which fixes the tensor's key

    def mix(x):
        x = (x * 0x9E3779B9) & 0xFFFFFFFF
        x = x ^ (x >> 15)
        x = (x * 0x6A09E667) & 0xFFFFFFFF
        return x ^ (x >> 13)

    def unmix(y):
        y = y ^ (y >> 13) ^ (y >> 26)
        y = y * pow(0x6A09E667, -1, 2 ** 32) % 2 ** 32
        y = y ^ (y >> 15) ^ (y >> 30)
        return y * pow(0x9E3779B9, -1, 2 ** 32) % 2 ** 32

    return mix((torch.arange(n, device="cuda") + unmix(first)) & 0xFFFFFFFF)


def encode(x, rnd, moment):
    """The documented codes and exponents of float32 values, on the device."""
    top, least = (15, 0) if moment == "m" else (31, 1)
    n = x.numel()
    pad = -n % 256
    mag = torch.nn.functional.pad(x.abs(), (0, pad)).view(torch.int32).long().view(-1, 256)
    rnd = torch.nn.functional.pad(rnd, (0, pad)).view(-1, 256)
    E = ((mag.amax(1, keepdim=True) + 0xFFFFF) >> 23).clamp(top + 1, 255)
    k = torch.where(mag > 0, (((mag + rnd) >> 20) - 8 * (E - top)).clamp(min=least), 0).view(-1)[:n]
    if moment == "m":
        k = k + torch.where(x < 0, 128, 0)
    return k.to(torch.uint8), E[:, 0].to(torch.uint8)


def decode(codes, exps, moment):
    top = 15 if moment == "m" else 31
    k = codes.int() & (127 if moment == "m" else 255)
    base = 8 * (exps.int() - top).repeat_interleave(256)[:k.numel()]
    x = torch.where(k > 0, ((k + base) << 20), 0).view(torch.float32)
    return torch.where(codes > 127, -x, x) if moment == "m" else x


def moments32(g, m, v, grad_scale):
    """m' and v' in float32, each operation rounded."""
    g = g * float(np.float32(grad_scale))
    return (m * float(np.float32(HYPER["beta1"])) + g * float(np.float32(1 - HYPER["beta1"])),
            v * float(np.float32(HYPER["beta2"])) + (g * g) * float(np.float32(1 - HYPER["beta2"])))


def check_large_param(got, p, g, m, v, step, grad_scale, half_ulp):
    """check_param's bound, on the device."""
    o = HYPER
    p, g, m, v = (x.double() for x in (p, g, m, v))
    g = g * grad_scale
    terms = (m * o["beta1"]).abs() + (g * (1 - o["beta1"])).abs()
    m, v = o["beta1"] * m + (1 - o["beta1"]) * g, o["beta2"] * v + (1 - o["beta2"]) * g * g
    rate = o["lr"] / (1 - o["beta1"] ** step) / ((v / (1 - o["beta2"] ** step)).sqrt() + o["eps"])
    want = p - o["lr"] * o["weight_decay"] * p - rate * m
    move = (rate * m).abs()
    tol = U * (3 * p.abs() + 3 * want.abs() + 12 * move + 4 * rate * terms) + half_ulp * want.abs() + 1e-37
    bad = ~((got.double() - want).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist())


@pytest.mark.parametrize("offset", [1, 3])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_past_the_caches(dtype, grad_dtype, bits, offset):
    item = {torch.float32: 4, torch.bfloat16: 2}
    element = item[dtype] + item[grad_dtype] + 2 * bits // 8
    sizes = SIZES + [(300 << 20) // element + 1357] + SIZES[::-1]
    print(f"case adamw large {dtype} {grad_dtype} bits={bits} offset={offset} n={max(sizes)}", flush=True)
    g = torch.Generator(device="cuda")
    g.manual_seed(offset)
    params = [make(n, dtype, g, 0.5, offset) for n in sizes]
    grads = [make(n, grad_dtype, g, 0.01, (offset * (i + 1)) % 5) for i, n in enumerate(sizes)]
    copies = [make(n, torch.bfloat16, g, 0.0, offset) for n in sizes] if dtype == torch.float32 else None
    opt = pr.AdamW(params, grads=grads, copies=copies, state_bits=bits, seed=SEED, steps=STEPS)
    for step in (STEPS + 1, STEPS + 2):
        for t in grads:
            t.normal_(generator=g).mul_(0.01)
        before = [p.clone() for p in params]
        states = [{k: x.clone() for k, x in s.items()} for s in opt.states]
        opt.step(grad_scale=0.5, **HYPER)
        values = opt.moments()
        torch.cuda.synchronize()
        for i, p in enumerate(params):
            s, was = opt.states[i], states[i]
            if bits == 32:
                m, v = was["m"], was["v"]
            else:
                m, v = (decode(was[k], was[k + "_exp"], k) for k in ("m", "v"))
            m1, v1 = moments32(grads[i].float(), m, v, 0.5)
            half_ulp = 0.0 if dtype == torch.float32 else 2.0 ** -7
            check_large_param(p, before[i], grads[i], m, v, step, 0.5, half_ulp)
            if copies:
                assert torch.equal(copies[i], p.bfloat16()), i
            if bits == 32:
                assert torch.equal(s["m"], m1) and torch.equal(s["v"], v1), i
                continue
            rnd = random_bits(p.numel(), i, step)
            for k, x, r, got in (("m", m1, rnd & 0xFFFFF, values[0][i]), ("v", v1, rnd >> 12, values[1][i])):
                codes, exps = encode(x, r, k)
                assert torch.equal(s[k], codes) and torch.equal(s[k + "_exp"], exps), (k, i)
                assert torch.equal(got.float(), decode(codes, exps, k)), (k, i)
            if i < len(SIZES):  # the device's forms of the coding against the oracle's
                n = p.numel()
                h = oadam.random_bits(n, i, SEED, step)
                assert np.array_equal(rnd.cpu().numpy().astype(np.uint64), h)
                hm, hv = f32_moments(host(grads[i]), host(m), host(v), HYPER, 0.5)
                for k, x, r in (("m", hm, h & np.uint64(0xFFFFF)), ("v", hv, h >> np.uint64(12))):
                    codes, exps = oadam.encode(x, r.astype(np.int64), k)
                    assert np.array_equal(s[k].cpu().numpy(), codes) and np.array_equal(s[k + "_exp"].cpu().numpy(), exps)
                if dtype == torch.float32:
                    check_param(host(p), host(before[i]), host(grads[i]), host(m), host(v), step, HYPER, 0.5)
    # nothing was written beside the tensors
    if dtype == torch.float32:
        for c in copies:
            assert not c._base[:offset].any() and not c._base[offset + c.numel():].any()
