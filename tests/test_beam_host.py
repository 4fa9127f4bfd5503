"""The entry points of beam search and distillation check their host-visible arguments before any launch (CPU only: no
call here reaches the GPU)."""

import ctypes as C
import math

import pytest

from tests.helpers import ensure_built

P = C.c_void_p(4096)
Q = C.c_void_p(1 << 30)


@pytest.fixture(scope="module")
def L():
    return ensure_built()


def _abi():
    from paper_2608_28726_amd import _abi as a
    return a


ROWS = [dict(dtype=3), dict(n=-1), dict(V=1), dict(stride=99), dict(logits=None), dict(T=None),
        dict(logits=C.c_void_p(4097))]


def top(L, **kw):
    a = _abi()
    x = dict(logits=P, dtype=a.PR_F32, n=4, V=100, stride=100, T=P, k=5, ids=P, logprob=P, lse=P, flags=P, ws=P, bytes=1 << 30)
    x.update(kw)
    return L.pr_top_logits(x["logits"], x["dtype"], x["n"], x["V"], x["stride"], x["T"], x["k"], x["ids"], x["logprob"],
                           x["lse"], x["flags"], x["ws"], x["bytes"], None)


@pytest.mark.parametrize("bad", ROWS + [dict(k=0), dict(k=257), dict(ids=None), dict(logprob=None)])
def test_top_refusals(L, bad):
    assert top(L, **bad) == _abi().PR_ERR_INVALID_ARG


def test_nothing_to_do(L):
    a = _abi()
    assert top(L, n=0) == a.PR_OK and top(L, n=(1 << 26) + 1) == a.PR_ERR_UNSUPPORTED
    assert select(L, n=0) == a.PR_OK
    assert reorder(L, [], n=3) == a.PR_OK and reorder(L, [(4096, 8, 8)], n=0) == a.PR_OK
    assert reorder(L, [(4096, 0, 8)], n=3) == a.PR_OK


def select(L, **kw):
    a = _abi()
    x = dict(logits=P, dtype=a.PR_BF16, n=4, B=4, V=100, stride=100, T=P, scores=P, done=None, token=0, k=4, best=P, parent=P,
             out_token=P, ws=P, bytes=1 << 30, out=True)
    x.update(kw)
    out = C.byref(a.BeamOut(x["best"], x["parent"], x["out_token"], None, None)) if x["out"] else None
    return L.pr_beam_select(x["logits"], x["dtype"], x["n"], x["B"], x["V"], x["stride"], x["T"], x["scores"], x["done"],
                            x["token"], x["k"], out, x["ws"], x["bytes"], None)


@pytest.mark.parametrize("bad", ROWS + [dict(B=0), dict(B=-1), dict(scores=None), dict(k=0), dict(k=257), dict(out=False),
                                        dict(best=None), dict(parent=None), dict(out_token=None), dict(ws=None),
                                        dict(bytes=8), dict(ws=C.c_void_p(4104))])
def test_select_refusals(L, bad):
    assert select(L, **bad) == _abi().PR_ERR_INVALID_ARG


def test_too_many(L):
    a = _abi()
    assert select(L, B=65) == a.PR_ERR_UNSUPPORTED
    assert select(L, n=1 << 22) == a.PR_ERR_UNSUPPORTED
    assert reorder(L, [(4096, 8, 8)], B=65) == a.PR_ERR_UNSUPPORTED
    assert reorder(L, [(4096, 8, 8)], n=1 << 30, B=2) == a.PR_ERR_UNSUPPORTED
    assert distill(L, n=(1 << 26) + 1) == a.PR_ERR_UNSUPPORTED


def reorder(L, states, n=3, B=2, parent=C.c_void_p(1 << 20), count=None):
    a = _abi()
    S = (a.BeamState * max(1, len(states)))(*[a.BeamState(p, b, s) for p, b, s in states])
    return L.pr_beam_reorder(S if states or count is None else None, len(states) if count is None else count, parent, n, B, None)


@pytest.mark.parametrize("states", [
    [(0, 8, 8)], [(4096, -1, 8)], [(4096, 9, 8)], [(4096, 8, 1 << 42)],
    [(4096, 8, 8), (4096, 8, 8)],            # the same state twice
    [(4096, 8, 8), (8192, 8, 8), (4096 + 47, 8, 8)],
    [(4096 + 8, 16, 16), (4096, 16, 16)],
    [(4096, 8, 32), (4096 + 4, 8, 32)],      # side by side, but over each other
    [(4096, 8, 32), (4096 + 28, 8, 32)],     # the second's row ends in the first's next
    [(4096, 8, 32), (4096 + 8, 8, 24)],      # other strides
    [((1 << 20) - 40, 8, 8)],                # the parents are among the rows
])
def test_reorder_refusals(L, states):
    assert reorder(L, states) == _abi().PR_ERR_INVALID_ARG


def test_other_reorder_refusals(L):
    a = _abi()
    assert reorder(L, [(4096, 8, 8)], B=0) == a.PR_ERR_INVALID_ARG
    assert reorder(L, [(4096, 8, 8)], n=-1) == a.PR_ERR_INVALID_ARG
    assert reorder(L, [(4096, 8, 8)], parent=None) == a.PR_ERR_INVALID_ARG
    assert reorder(L, [], count=1) == a.PR_ERR_INVALID_ARG
    assert reorder(L, [], count=-1) == a.PR_ERR_INVALID_ARG
    assert L.pr_stream_reorder(None, P, P, 1, 1, None) == a.PR_ERR_INVALID_ARG


def distill(L, **kw):
    a = _abi()
    x = dict(logits=P, dtype=a.PR_BF16, n=4, V=100, stride=100, ids=P, logq=P, k=5, top_stride=5, T=P, w=P, params=None, loss=P,
             out=None, grad=Q, gstride=100, ws=P, bytes=1 << 30)
    x.update(kw)
    params = None if x["params"] is None else C.byref(a.DistillParams(*x["params"]))
    return L.pr_distill_loss(x["logits"], x["dtype"], x["n"], x["V"], x["stride"], x["ids"], x["logq"], x["k"],
                             x["top_stride"], x["T"], x["w"], params, x["loss"], x["out"], x["grad"], x["gstride"],
                             x["ws"], x["bytes"], None)


@pytest.mark.parametrize("bad", ROWS + [
    dict(ids=None), dict(logq=None), dict(w=None), dict(w=None, k=0), dict(loss=None), dict(k=-1), dict(k=257, top_stride=257),
    dict(top_stride=4), dict(params=(3, 1.0)), dict(params=(-1, 1.0)), dict(params=(0, math.nan)), dict(gstride=99),
    dict(grad=C.c_void_p((1 << 30) + 1)), dict(ws=None), dict(bytes=8), dict(ws=C.c_void_p(4104)),
    dict(grad=P, gstride=101), dict(grad=C.c_void_p(4096 + 400))])
def test_distill_refusals(L, bad):
    assert distill(L, **bad) == _abi().PR_ERR_INVALID_ARG


def test_defaults_and_workspaces(L):
    a = _abi()
    p = a.DistillParams()
    L.pr_distill_params_default(C.byref(p))
    assert (p.tail, p.grad_scale) == (a.PR_TAIL_REST, 1.0)
    L.pr_distill_params_default(None)
    for n in (0, -3):
        assert L.pr_distill_loss_workspace(a.PR_F32, n, 1000, 64) == 0
        assert L.pr_top_logits_workspace(a.PR_F32, n, 1000, 64) == 0
        assert L.pr_beam_select_workspace(a.PR_F32, n, 4, 1000, 64) == 0
    assert L.pr_distill_loss_workspace(a.PR_BF16, 17904, 151936, 64) <= 128 * 17904


def test_bindings_refuse_host_tensors():
    import torch

    import paper_2608_28726_amd as pr
    z, f = torch.zeros(2, 8), torch.zeros(2)
    ids, parent = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises(ValueError):
        pr.top_logits(z, 2)
    with pytest.raises(ValueError):
        pr.beam_select(z, torch.zeros(1, 2))
    with pytest.raises(ValueError):
        pr.beam_reorder([z], parent)
    with pytest.raises(ValueError):
        pr.distill_loss(z, ids, torch.zeros(2, 3), f, f)
    with pytest.raises(ValueError):
        pr.distill_loss(z, ids, torch.zeros(2, 3), f, f, tail="all")
