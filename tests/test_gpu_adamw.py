"""The AdamW step over many tensors: HIP path vs the oracle.

Tolerances. m' and v' are two products and a sum in float32: off by at most
3 x 2^-24 of the larger of their terms. p' adds p's product (2^-24 |p|), the
sum (2^-24 |p'|) and the update's error: m' and v' 's, and at most 6 roundings
of 2^-24 each. 8-bit codes follow from m' and v' in float32, whose operations
are written out and not fused, so numpy's float32 gives the same bits.
"""

import math

import numpy as np
import pytest
import torch

import paper_2608_28726_amd as pr
from oracle import adamw as oadam
from paper_2608_28726_amd import _abi
from tests.gpu_common import require_gpu

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HYPER = dict(lr=0.01, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


SIZES = [1, 2, 3, 4, 5, 255, 256, 257, 1023, 4095, 4096, 4097, 9001, 70000]


def tensors(sizes, dtype, seed, scale=1.0, offset=0):
    """A tensor per size, each starting `offset` elements into a buffer of its own."""
    rng = np.random.default_rng(seed)
    out = []
    for n in sizes:
        buf = torch.zeros(n + offset + 3, dtype=dtype, device="cuda")
        t = buf[offset:offset + n]
        t.copy_(torch.tensor(rng.normal(0, scale, n) * np.exp(rng.normal(0, 1, n))))
        out.append(t)
    return out


def host(t):
    return t.detach().float().cpu().numpy()


def f32_moments(g, m, v, o, grad_scale):
    f = np.float32
    g = (g * f(grad_scale)).astype(f)
    m1 = (m * f(o["beta1"])).astype(f) + (g * f(1 - o["beta1"])).astype(f)
    v1 = (v * f(o["beta2"])).astype(f) + ((g * g).astype(f) * f(1 - o["beta2"])).astype(f)
    return m1.astype(f), v1.astype(f)


def check_param(got, p, g, m, v, step, o, grad_scale, half_ulp=0.0):
    """got against the float64 step from the same float32 state."""
    want, m64, v64 = oadam.adamw(p, g, m, v, step, grad_scale=grad_scale, **o)
    move = np.abs(want - p.astype(np.float64) * (1 - o["lr"] * o["weight_decay"]))
    # m' may cancel: its error is of its terms' size
    terms = np.abs(m * o["beta1"]) + np.abs(g * grad_scale * (1 - o["beta1"]))
    rate = o["lr"] / (1 - o["beta1"] ** step) / (np.sqrt(v64 / (1 - o["beta2"] ** step)) + o["eps"])
    tol = U * (3 * np.abs(p) + 3 * np.abs(want) + 12 * move + 4 * rate * terms) + half_ulp * np.abs(want) + 1e-37
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.flatnonzero(bad)[:4], got[bad][:4], want[bad][:4])


@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("given", [True, False])
def test_float32_parameters(bits, grad_dtype, offset, given):
    print(f"case adamw f32 bits={bits} {grad_dtype} offset={offset} given={given}", flush=True)
    params = tensors(SIZES, torch.float32, 1, 0.5, offset)
    copies = [torch.zeros_like(p, dtype=torch.bfloat16) for p in params]
    grads = tensors(SIZES, grad_dtype, 2, 1e-2, offset)
    opt = pr.AdamW(params, grads=None if given else grads, copies=copies, state_bits=bits, seed=9)
    for step in range(1, 4):
        before = [host(p) for p in params]
        if bits == 32:
            m = [host(s["m"]) for s in opt.states]
            v = [host(s["v"]) for s in opt.states]
        else:
            m, v = ([oadam.decode(s[k].cpu().numpy(), s[k + "_exp"].cpu().numpy(), k).astype(np.float32)
                     for s in opt.states] for k in ("m", "v"))
        for i, g in enumerate(grads):
            g.copy_(torch.tensor(np.random.default_rng(100 * step + i).normal(0, 0.01, g.numel())))
        opt.step(grads=grads if given else None, grad_scale=0.5, **HYPER)
        torch.cuda.synchronize()
        got_m, got_v = opt.moments()
        for i, p in enumerate(params):
            g = host(grads[i])
            check_param(host(p), before[i], g, m[i], v[i], step, HYPER, 0.5)
            assert torch.equal(copies[i], p.bfloat16())
            m1, v1 = f32_moments(g, m[i], v[i], HYPER, 0.5)
            if bits == 32:
                assert np.array_equal(host(opt.states[i]["m"]), m1) and np.array_equal(host(opt.states[i]["v"]), v1)
                continue
            bits32 = oadam.random_bits(p.numel(), i, 9, step)
            for k, x, rnd, got in (("m", m1, bits32 & np.uint64(0xFFFFF), got_m), ("v", v1, bits32 >> np.uint64(12), got_v)):
                codes, exps = oadam.encode(x, rnd.astype(np.int64), k)
                assert np.array_equal(opt.states[i][k].cpu().numpy(), codes), (k, i)
                assert np.array_equal(opt.states[i][k + "_exp"].cpu().numpy(), exps), (k, i)
                assert np.array_equal(host(got[i]), oadam.decode(codes, exps, k).astype(np.float32)), (k, i)


@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("bits", [32, 8])
def test_bfloat16_parameters(bits, grad_dtype):
    """A bfloat16 parameter goes to one of the two neighbours of the float32 step, up with the probability of the
    part it loses: its bits plus 16 random ones."""
    params = tensors(SIZES, torch.bfloat16, 3, 0.5)
    grads = tensors(SIZES, grad_dtype, 4, 1e-2)
    before = [host(p) for p in params]
    opt = pr.AdamW(params, grads=grads, state_bits=bits, seed=77, steps=4)
    opt.step(**HYPER)
    torch.cuda.synchronize()
    assert opt.steps == 5
    for i, p in enumerate(params):
        zero = np.zeros(p.numel(), np.float32)
        check_param(host(p), before[i], host(grads[i]), zero, zero, 5, HYPER, 1.0, half_ulp=2.0 ** -7)
    # on average nothing is lost: many elements of one value, each moved by a sixteenth of its spacing
    n = 1 << 16
    p = torch.full((n,), 1.0, dtype=torch.bfloat16, device="cuda")
    g = torch.full((n,), -1.0, device="cuda")
    o = pr.AdamW([p], grads=[g], seed=5)
    o.step(lr=2.0 ** -11, beta1=0.0, beta2=0.0, eps=0.0, weight_decay=0.0)
    torch.cuda.synchronize()
    up = float((p.double() - 1.0).mean())
    # spacing 2^-7 above 1, probability 1/16 each: standard deviation of the mean 2^-7 x 0.242 / 256
    assert abs(up - 2.0 ** -11) < 5 * 2.0 ** -7 * 0.242 / 256 and set(p.double().unique().tolist()) == {1.0, 1 + 2.0 ** -7}


@pytest.mark.parametrize("count", [1, 399, 400, 401, 900])
def test_many_tensors(count):
    """Lists that take one launch and several, empty tensors and tensors without a gradient among them."""
    sizes = [(7 * i) % 513 for i in range(count)]
    params = [torch.full((k,), 1.0, device="cuda") for k in sizes]
    grads = [torch.full((k,), 0.25, device="cuda") if i % 5 != 3 else None for i, k in enumerate(sizes)]
    opt = pr.AdamW(params, state_bits=8)
    opt.step(lr=0.125, weight_decay=0.0, grads=grads)
    torch.cuda.synchronize()
    m, v = opt.moments()
    for i, p in enumerate(params):
        # the first step moves by lr g / (|g| + eps)
        want = 1.0 if grads[i] is None else 0.875
        assert p.numel() == 0 or abs(float(p.min()) - want) < 1e-6 and abs(float(p.max()) - want) < 1e-6, i
        assert bool((m[i] == 0).all()) == (grads[i] is None or p.numel() == 0)


@pytest.mark.parametrize("bits", [32, 8])
def test_nonfinite_gradients(bits):
    """A NaN or an infinity stays in its element (its block, for 8-bit states); zeros stay zero."""
    p = torch.full((1024,), 2.0, device="cuda")
    g = torch.zeros(1024, device="cuda")
    g[300] = math.nan
    g[600] = math.inf
    opt = pr.AdamW([p], grads=[g], state_bits=bits)
    opt.step(lr=0.1, weight_decay=0.0)
    torch.cuda.synchronize()
    bad = torch.isnan(p).nonzero()[:, 0].tolist()
    assert bad == [300, 600]
    assert bool((p[torch.tensor([0, 299, 301, 1023])] == 2.0).all())
    m, v = opt.moments()
    if bits == 8:
        assert torch.isnan(m[0][256:768].float()).all() and torch.isnan(v[0][256:768].float()).all()
        assert bool((m[0][:256] == 0).all()) and bool((v[0][768:] == 0).all())
    else:
        assert math.isnan(float(m[0][300])) and float(m[0][600]) == math.inf


def test_eight_bit_training_follows_the_32_bit_one():
    """A least-squares problem: with 8-bit states the loss falls as it does with 32-bit ones (within 20 %), from the
    same start over 300 steps."""
    torch.manual_seed(0)
    A = torch.randn(256, 64, device="cuda") / 8
    target = A @ torch.randn(64, 20, device="cuda")
    losses = []
    for bits in (32, 8):
        w = torch.zeros(64, 20, device="cuda")
        opt = pr.AdamW([w], state_bits=bits, seed=3)
        for _ in range(300):
            r = A @ w - target
            opt.step(lr=0.02, weight_decay=0.0, grads=[(A.t() @ r) / 256])
        losses.append(float((A @ w - target).square().mean()))
    first = float(target.square().mean())
    assert losses[0] < 0.02 * first and losses[1] < 0.02 * first + 1.2 * losses[0], (first, losses)


def test_more_elements_than_a_launch():
    """17.2e9 elements, more than 2^32 threads take 4 each: several launches, and element offsets past 2^34. Random
    numbers repeat after 2^32 elements, and so does all else here."""
    n = (1 << 34) + 4096 + 77
    if torch.cuda.mem_get_info()[0] < 115 << 30:
        pytest.skip("needs 103 GB of device memory")
    print(f"case adamw n={n}", flush=True)
    p = torch.full((n,), 1.0, dtype=torch.bfloat16, device="cuda")
    g = torch.full((n,), -0.25, dtype=torch.bfloat16, device="cuda")
    opt = pr.AdamW([p], grads=[g], state_bits=8, seed=5)
    # the first step moves every element by lr, twice the spacing of bfloat16 above 1
    opt.step(lr=2.0 ** -6, eps=0.0, weight_decay=0.0)
    torch.cuda.synchronize()
    s = opt.states[0]
    k = 70000
    m, v = f32_moments(np.full(k, -0.25, np.float32), np.zeros(k, np.float32), np.zeros(k, np.float32),
                       dict(beta1=0.9, beta2=0.999), 1.0)
    bits = oadam.random_bits(k, 0, 5, 1)
    for name, x, rnd in (("m", m, bits & np.uint64(0xFFFFF)), ("v", v, bits >> np.uint64(12))):
        codes, exps = oadam.encode(x, rnd.astype(np.int64), name)
        assert np.array_equal(s[name][:k].cpu().numpy(), codes)
        assert np.array_equal(s[name + "_exp"][:k // 256].cpu().numpy(), exps[:k // 256])
    assert float(p[:k].min()) >= 1.0 + 2.0 ** -7 and float(p[:k].max()) <= 1.0 + 3 * 2.0 ** -7
    for t, period in ((p, 1 << 32), (s["m"], 1 << 32), (s["v"], 1 << 32), (s["m_exp"], 1 << 24), (s["v_exp"], 1 << 24)):
        for a in range(period, t.numel(), period):
            part = t[a:a + period]
            assert torch.equal(part, t[:part.numel()]), (period, a)
    del p, g, opt, s, t, part
    torch.cuda.empty_cache()


def test_step_on_another_stream_and_in_a_graph():
    sizes = [5, 300, 70001]
    runs = []
    for mode in ("eager", "stream", "graph"):
        params = tensors(sizes, torch.float32, 8)
        grads = tensors(sizes, torch.bfloat16, 9)
        opt = pr.AdamW(params, grads=grads, state_bits=8, seed=2)
        torch.cuda.synchronize()
        if mode == "eager":
            opt.step(**HYPER)
        elif mode == "stream":
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                opt.step(**HYPER)
            s.synchronize()
        else:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                opt.step(**HYPER)
            g.replay()
        torch.cuda.synchronize()
        runs.append([*params, *[s[k] for s in opt.states for k in s]])
    for other in runs[1:]:
        for a, b in zip(runs[0], other):
            assert torch.equal(a, b)


def test_refusals():
    p = torch.zeros(300, device="cuda")
    g = torch.zeros(300, device="cuda")
    u8 = lambda k: torch.zeros(k, dtype=torch.uint8, device="cuda")  # noqa: E731
    bad = [dict(params=[]), dict(params=[p.cpu()]), dict(params=[p, p.bfloat16()]), dict(params=[p.half()]),
           dict(params=[torch.zeros(4, 4, device="cuda").t()]), dict(grads=[g, g]), dict(grads=[g[:5]]), dict(grads=[None]),
           dict(grads=[g.double()]), dict(state_bits=16), dict(copies=[p]), dict(copies=[torch.zeros(3, device="cuda").bfloat16()]),
           dict(states=[]), dict(states=[{"m": p}]), dict(states=[{"m": p, "v": p.bfloat16()}]),
           dict(state_bits=8, states=[{"m": u8(300), "v": u8(300), "m_exp": u8(2), "v_exp": u8(1)}]),
           dict(params=[p.bfloat16()], copies=[p.bfloat16()])]
    for kw in bad:
        with pytest.raises((ValueError, TypeError)):
            pr.AdamW(**{"params": [p], **kw})
    opt = pr.AdamW([p])
    with pytest.raises(ValueError):
        opt.step(lr=0.1)
    with pytest.raises(ValueError):
        opt.step(lr=0.1, grads=[None])
    opt = pr.AdamW([p], grads=[g])
    for kw in (dict(lr=math.nan), dict(lr=0.1, beta1=1.0), dict(lr=0.1, beta2=-0.1), dict(lr=0.1, eps=-1.0),
               dict(lr=0.1, grad_scale=math.inf)):
        with pytest.raises(pr.ProuterError):
            opt.step(**kw)
    assert opt.steps == 0
    with pytest.raises(ValueError):
        opt.step(lr=0.1, grads=[g.bfloat16()])
    eight = pr.AdamW([p], state_bits=8)
    with pytest.raises(ValueError):
        eight.moments(out=(torch.zeros(512, dtype=torch.bfloat16, device="cuda"), torch.zeros(300, device="cuda")))


def test_closed_and_replanned():
    """A closed optimizer takes no step and no moments (a plan made anew for moments once took the gradients' buffers
    for the parameters' type). Moments before the first step leave later steps as they are."""
    n = 3001
    for bits in (8, 32):
        p, g = torch.ones(n, device="cuda"), torch.ones(n, dtype=torch.bfloat16, device="cuda")
        opt = pr.AdamW([p], grads=[g], state_bits=bits)
        opt.step(lr=0.125)
        opt.close()
        opt.close()
        for call in (opt.moments, lambda: opt.step(lr=0.125), lambda: opt.step(lr=0.125, grads=[g.float()])):
            with pytest.raises(ValueError):
                call()
        assert opt.steps == 1
    for grad_dtype in (torch.float32, torch.bfloat16):
        runs = []
        for first in (False, True):
            p, g = torch.ones(n, device="cuda"), torch.linspace(-1, 1, n, device="cuda").to(grad_dtype)
            opt = pr.AdamW([p], state_bits=8, seed=4)
            if first:
                m, v = opt.moments()
                assert bool((m[0] == 0).all()) and bool((v[0] == 0).all())
            for _ in range(2):
                opt.step(lr=0.125, grads=[g])
                opt.moments()
            torch.cuda.synchronize()
            runs.append([p, *opt.states[0].values()])
        for a, b in zip(*runs):
            assert torch.equal(a, b)


def test_first_step_captured_after_moments():
    """A plan that moments() made serves a first step with gradients of the parameters' type, also in a graph."""
    n = 3001
    p, g = torch.ones(n, device="cuda"), torch.linspace(-1, 1, n, device="cuda")
    other = p.clone()
    opt, eager = pr.AdamW([p], state_bits=8), pr.AdamW([other], state_bits=8)
    opt.moments()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step(lr=0.125, grads=[g])
    graph.replay()
    eager.step(lr=0.125, grads=[g])
    torch.cuda.synchronize()
    assert torch.equal(p, other)


def test_no_plan_on_another_device(monkeypatch):
    """With another device current, calls are refused before they make a plan, which would lie on that device."""
    p, g = torch.ones(300, device="cuda"), torch.ones(300, device="cuda")
    opt = pr.AdamW([p], state_bits=8)
    made = []
    create = _abi.lib().pr_adamw_create
    with monkeypatch.context() as patch:
        patch.setattr(torch.cuda, "current_device", lambda: p.device.index + 1)
        patch.setattr(_abi.lib(), "pr_adamw_create", lambda *a: made.append(a) or create(*a))
        for call in (opt.moments, lambda: opt.step(lr=0.125, grads=[g])):
            with pytest.raises(ValueError):
                call()
    assert not made and opt.steps == 0
    opt.step(lr=0.125, weight_decay=0.0, grads=[g])
    assert abs(float(p[0]) - 0.875) < 1e-6




def test_replaced_storages():
    """What a step writes to stays allocated, and is what was checked, when a parameter, gradient or state is given
    another storage afterwards."""
    n = 1 << 20
    big = [torch.ones(n, device="cuda") for _ in range(2)]
    wide = torch.full((2 * n,), 3.0, device="cuda")
    for bound in (True, False):
        p, g = big[0].clone(), big[1].clone()
        opt = pr.AdamW([p], grads=[g] if bound else None, copies=[p.bfloat16()])
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        kept, p.data = p.detach(), wide
        opt.states[0]["v"] = None
        opt.copies[0] = None
        if bound:
            g.data = torch.zeros(2, device="cuda")
        assert torch.cuda.memory_allocated() >= before
        # the step goes to what was given, and to nothing else
        del opt.params[:]
        opt.step(lr=0.125, weight_decay=0.0, grads=None if bound else [g])
        torch.cuda.synchronize()
        assert bool(((kept - 0.875).abs() < 1e-6).all()) and bool((wide == 3.0).all())
        del kept, opt


def decay_case(n, dtype, seed):
    """Parameters of size about 1 with states that move each by an update of its own, 1e-6 wide: many times the
    spacing of float32, so that roundings to nearest average out."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    p = (torch.rand(n, generator=g, device="cuda") + 0.5).to(dtype)
    m = torch.empty(n, device="cuda").normal_(generator=g)
    v = torch.ones(n, device="cuda")
    grad = torch.empty(n, device="cuda").normal_(generator=g)
    return p, grad, m, v


@pytest.mark.parametrize("weight_decay", [0.01, 0.1, 0.2])
@pytest.mark.parametrize("eps", [1e-8, 0.0])
def test_weight_decay_at_small_rates(weight_decay, eps):
    """lr weight_decay far below float32's spacing at 1: on average every parameter decays by it. A rounding moves
    p'/p by 2^-24 at most, 3.5e-8 in the mean square; the mean of 2^20 of them is within 5 x 3.5e-8 / 2^10 of 0."""
    n, o = 1 << 20, dict(lr=1e-6, beta1=0.9, beta2=0.999, eps=eps, weight_decay=weight_decay)
    p, grad, m, v = decay_case(n, torch.float32, 31)
    before = [host(x) for x in (p, grad, m, v)]
    pr.AdamW([p], grads=[grad], states=[dict(m=m, v=v)], steps=500).step(**o)
    torch.cuda.synchronize()
    want, _, _ = oadam.adamw(*before, 501, **o)
    off = float(np.mean((host(p).astype(np.float64) - want) / before[0]))
    assert abs(off) <= 5 * 3.5e-8 / 2 ** 10, (off, o["lr"] * weight_decay)


def test_weight_decay_of_bfloat16_parameters_at_small_rates():
    """The float32 step that a bfloat16 parameter is rounded from holds the decay: with the documented random bits the
    stochastic rounding gives the same 16 bits. The update is off by about 4e-7 of 1e-6, so the float32 step differs
    from the float64 one's nearest in 1 of 10^5 elements, and its rounding in 1 of 2^16 of those: none of 2^24."""
    n, o = 1 << 24, dict(lr=1e-6, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01)
    p, grad, m, v = decay_case(n, torch.bfloat16, 32)
    before = [host(x) for x in (p, grad, m, v)]
    pr.AdamW([p], grads=[grad], states=[dict(m=m, v=v)], steps=500, seed=6).step(**o)
    torch.cuda.synchronize()
    want, _, _ = oadam.adamw(*before, 501, **o)
    bits = want.astype(np.float32).view(np.uint32) + (oadam.random_bits(n, 0, 6, 501) & np.uint64(0xFFFF)).astype(np.uint32)
    off = int((p.view(torch.int16).cpu().numpy().view(np.uint16) != (bits >> np.uint32(16)).astype(np.uint16)).sum())
    assert off <= 1, off


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("weight_decay", [0.0, 0.1])
def test_infinite_parameters_stay(dtype, weight_decay):
    p = torch.tensor([math.inf, -math.inf, 1.0, math.nan], device="cuda").to(dtype)
    pr.AdamW([p], grads=[torch.full((4,), 0.5, device="cuda")]).step(lr=2.0 ** -6, weight_decay=weight_decay)
    torch.cuda.synchronize()
    assert p[:2].tolist() == [math.inf, -math.inf] and 0.97 < float(p[2]) < 1.0 and math.isnan(float(p[3]))


def test_small_eps_beside_a_large_correction():
    """eps = 1e-12 with beta2 so near 1 that c2 sqrt(v) counts beside it for v below 2^-126."""
    o = dict(lr=1.0, beta1=0.9, beta2=1 - 2.0 ** -40, eps=1e-12, weight_decay=0.0)
    z = np.zeros(5, np.float32)
    m = np.array([1e-12, -3e-12, 2e-12, 1e-13, 0.0], np.float32)
    v = np.array([1e-38, 5e-39, 1.1e-38, 2e-39, 1e-38], np.float32)
    p, grad = torch.zeros(5, device="cuda"), torch.zeros(5, device="cuda")
    pr.AdamW([p], grads=[grad], states=[dict(m=torch.tensor(m, device="cuda"), v=torch.tensor(v, device="cuda"))]).step(**o)
    torch.cuda.synchronize()
    check_param(host(p), z, z, m, v, 1, o, 1.0)


def test_moments_of_32_bit_states_take_no_buffers():
    """32-bit states are returned themselves: buffers that would be left as they are get refused."""
    p = torch.zeros(300, device="cuda")
    opt = pr.AdamW([p])
    out = tuple(torch.zeros(512, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    with pytest.raises(ValueError):
        opt.moments(out=out)
    assert opt.moments()[0][0].data_ptr() == opt.states[0]["m"].data_ptr()
