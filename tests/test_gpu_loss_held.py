"""The policy loss on rows that a workgroup holds, as a training step calls it: with a reference and a KL term, its
gradient in the logits' place or at another stride, on a stream, in a captured graph, and over more rows than a
workgroup lists. Against plain float64 operations on the device.

Tolerances as in test_gpu_loss: l is off by L_ABS. dloss/dl = w (-ratio A - kl_coef (exp(d) - 1)) moves by
w (ratio |A| + kl_coef exp(d)) times that, and its exponentials are off by two roundings, less than L_ABS; |delta - p|
is at most 1, and p's error adds 2^-21 of the coefficient.
"""

import math

import pytest
import torch

import paper_2608_28726_amd as pr
from paper_2608_28726_amd import _abi
from tests import test_gpu_loss as base
from tests.gpu_common import require_gpu
from tests.test_gpu_loss import L_ABS, near

pytestmark = pytest.mark.gpu

KL, LO, HI, SCALE = 0.07, 0.2, 0.3, 2.5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


# Rows of both sizes that are held: a row for each workgroup, several of them, odd lengths
SHAPES = [(70, 40000, torch.float32), (600, 32000, torch.float32), (600, 50257, torch.bfloat16),
          (600, 28007, torch.bfloat16), (300, 70001, torch.float32), (300, 151936, torch.bfloat16)]


def batch(n, V, dtype, pad=0, start=0, seed=1):
    """Rows of stride V + pad, `start` elements into a buffer, a third of them not counting (and holding NaN); the
    arguments of the loss; each row's log-prob in 64 bits."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + n + V)
    flat = torch.empty(n * (V + pad) + start + 8, device="cuda").normal_(generator=g).mul_(3.0).to(dtype)
    logits = flat[start:start + n * (V + pad)].view(n, V + pad)[:, :V]
    ids = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    T = torch.rand(n, generator=g, device="cuda") + 0.5
    w = torch.rand(n, generator=g, device="cuda") + 0.1
    w[torch.rand(n, generator=g, device="cuda") < 0.3] = 0.0
    on = w != 0
    A = torch.empty(n, device="cuda").normal_(generator=g)
    l = torch.log_softmax(logits.double() / T[:, None].double(), 1).gather(1, ids[:, None].long())[:, 0]
    delta = torch.empty(n, device="cuda").normal_(generator=g).mul_(0.3)
    for edge in (1 - LO, 1 + HI):
        delta = torch.where((delta.exp() - edge).abs() < 2e-3, delta + 0.01, delta)
    old = (l - delta).float()
    ref = (l + torch.empty(n, device="cuda").normal_(generator=g).mul_(0.4)).float()
    logits[~on] = math.nan
    return flat, logits, (ids, T, w, A, old, ref), torch.where(on, l, 0.0)


def loss(logits, args, **kw):
    return pr.policy_loss(logits, *args, clip_low=LO, clip_high=HI, kl_coef=KL, grad_scale=SCALE, **kw)


def check(got, logits, args, l):
    """got against float64 operations on `logits`."""
    ids, T, w, A, old, ref = args
    on = w != 0
    zero = torch.zeros_like(l)
    ratio = torch.exp(l - old.double())
    d = ref.double() - l
    free, held = ratio * A, ratio.clamp(1 - LO, 1 + HI) * A
    clipped = on & (free > held)
    kl = torch.expm1(d) - d
    reach = torch.where(on, w * (ratio * A.abs() + KL * d.exp()), zero)
    terms = torch.where(on, w * (KL * kl - torch.minimum(free, held)), zero)
    assert torch.equal(got["flags"], torch.where(on, torch.where(clipped, pr.FLAG_CLIPPED, 0), pr.FLAG_MASKED).int())
    near("logprob", got["logprob"].cpu(), l.cpu(), L_ABS)
    near("ratio", got["ratio"].cpu(), torch.where(on, ratio, zero).cpu(), 0.0, 2 * L_ABS)
    near("kl", got["kl"].cpu(), torch.where(on, kl, zero).cpu(), L_ABS * (1 + d.exp()).cpu().numpy())
    near("loss", got["loss"].cpu(), [float(terms.sum())], 2 * L_ABS * float(reach.sum()))
    coef = torch.where(on, SCALE * w * (torch.where(clipped, zero, -free) - KL * torch.expm1(d)) / T, zero)[:, None]
    want = -torch.softmax(logits.double() / T[:, None].double(), 1)
    want.scatter_add_(1, ids[:, None].long(), torch.ones_like(want[:, :1]))
    want = torch.where(on[:, None], want * coef, 0.0)
    half_ulp = 2.0 ** -8 if logits.dtype == torch.bfloat16 else 2.0 ** -24
    allowed = coef.abs() * 2.0 ** -21 + 2 * L_ABS * SCALE * (reach / T)[:, None] + half_ulp * 1.01 * want.abs() + 1e-38
    bad = ~((got["grad"].double() - want).abs() <= allowed)
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:3].tolist())


def same(a, b):
    for k in ("loss", "logprob", "ratio", "kl", "flags", "grad"):
        assert torch.equal(a[k], b[k]), k


@pytest.mark.parametrize("pad,start", [(0, 0), (5, 3)])
@pytest.mark.parametrize("n,V,dtype", SHAPES)
def test_reference_and_in_place(n, V, dtype, pad, start):
    """With a KL term against float64; then the gradient in the logits' place, to the bit, and nothing beside it."""
    print(f"case held n={n} V={V} {dtype} pad={pad} start={start}", flush=True)
    flat, logits, args, l = batch(n, V, dtype, pad, start)
    before = flat.clone()
    got = loss(logits, args)
    check(got, logits, args, l)
    assert torch.equal(flat.view(torch.uint8), before.view(torch.uint8))
    again = loss(logits, args, grad=logits)
    torch.cuda.synchronize()
    assert again["grad"] is logits
    same(again, got)
    inside = torch.zeros(flat.shape, dtype=torch.bool, device="cuda")
    inside[start:start + n * (V + pad)].view(n, V + pad)[:, :V] = True
    assert torch.equal(flat[~inside], before[~inside])


@pytest.mark.parametrize("n,V,dtype", SHAPES)
def test_gradient_elsewhere(n, V, dtype):
    """A gradient whose rows sit otherwise than the logits' relative to 16 bytes, with what lies between left alone."""
    _, logits, args, l = batch(n, V, dtype, 2, 1)
    flat = torch.full((n * (V + 3) + 9,), 7.0, dtype=dtype, device="cuda")
    grad = flat[1:1 + n * (V + 3)].view(n, V + 3)[:, 2:V + 2]
    got = loss(logits, args, grad=grad)
    check(got, logits, args, l)
    grad.fill_(7.0)
    assert bool((flat == 7.0).all())


@pytest.mark.parametrize("n,V,dtype", SHAPES)
def test_stream_and_graph(n, V, dtype):
    """On another stream with a workspace full of NaN, and captured with the gradient in the place of a copy of the
    logits: every replay gives the eager call's bits, with new logits in between."""
    _, logits, args, _ = batch(n, V, dtype)
    ws = torch.full((int(_abi.lib().pr_policy_loss_workspace(pr._dtype_code(logits), n, V)),), 255, dtype=torch.uint8,
                    device="cuda")
    got = loss(logits, args)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = loss(logits, args, workspace=ws)
        place = torch.empty_like(logits)
        loss(logits, args, grad=place)  # a captured call's allocations have been made once
    side.synchronize()
    same(other, got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        torch.add(logits, 0.0, out=place)
        held = loss(place, args, grad=place)
    for k in range(3):
        logits.copy_(logits.roll(k + 1, 1))
        eager = loss(logits, args)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        same(held, eager)


@pytest.mark.parametrize("n,V,dtype", [(65601, 36008, torch.bfloat16), (65537, 18001, torch.float32),
                                       (65601, 68200, torch.bfloat16)])
def test_more_rows_than_are_listed(n, V, dtype):
    """Batches whose rows are dealt out by row, several to a workgroup, those that do not count among them."""
    if torch.cuda.mem_get_info()[0] < 64 << 30:
        pytest.skip("needs 60 GB of device memory")
    base.test_policy_many_rows(n, V, dtype, 0)
    torch.cuda.empty_cache()
