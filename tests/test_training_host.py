"""The training entry points check their host-visible arguments before any
launch (CPU only: no call here reaches the GPU)."""

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


def policy(L, **kw):
    a = _abi()
    x = dict(logits=P, dtype=a.PR_BF16, n=4, V=100, stride=100, ids=P, T=P, w=P, A=P, old=P, ref=None, params=None, loss=P,
             out=None, grad=Q, gstride=100, ws=P, bytes=1 << 20)
    x.update(kw)
    params = None if x["params"] is None else C.byref(a.PolicyParams(*x["params"]))
    return L.pr_policy_loss(x["logits"], x["dtype"], x["n"], x["V"], x["stride"], x["ids"], x["T"], x["w"], x["A"],
                            x["old"], x["ref"], params, x["loss"], x["out"], x["grad"], x["gstride"], x["ws"],
                            x["bytes"], None)


def preference(L, **kw):
    a = _abi()
    x = dict(logits=P, dtype=a.PR_F32, n=4, V=100, stride=100, ids=P, T=P, w=P, off=P, pairs=2, ref=None, params=None,
             loss=P, out=None, grad=Q, gstride=100, ws=P, bytes=1 << 20)
    x.update(kw)
    params = None if x["params"] is None else C.byref(a.PreferenceParams(*x["params"]))
    return L.pr_preference_loss(x["logits"], x["dtype"], x["n"], x["V"], x["stride"], x["ids"], x["T"], x["w"], x["off"],
                                x["pairs"], x["ref"], params, x["loss"], x["out"], x["grad"], x["gstride"], x["ws"],
                                x["bytes"], None)


ROWS = [dict(dtype=3), dict(n=-1), dict(V=1), dict(stride=99), dict(logits=None), dict(ids=None), dict(T=None), dict(w=None),
        dict(loss=None), dict(gstride=99), dict(grad=C.c_void_p((1 << 30) + 1)), dict(ws=None), dict(bytes=8),
        dict(ws=C.c_void_p(4104)), dict(grad=P, gstride=101), dict(grad=C.c_void_p(4096 + 400)),
        dict(stride=1 << 40, gstride=1 << 40)]


@pytest.mark.parametrize("bad", ROWS + [dict(A=None), dict(old=None), dict(params=(1.1, 0.2, 0, 1)),
                                        dict(params=(-0.1, 0.2, 0, 1)), dict(params=(0.2, -1.0, 0, 1)),
                                        dict(params=(0.2, math.nan, 0, 1)), dict(params=(0.2, 0.2, -1.0, 1)),
                                        dict(params=(0.2, 0.2, math.inf, 1)), dict(params=(0.2, 0.2, 0.1, 1)),
                                        dict(params=(0.2, 0.2, 0, math.nan))])
def test_policy_refusals(L, bad):
    assert policy(L, **bad) == _abi().PR_ERR_INVALID_ARG


@pytest.mark.parametrize("bad", ROWS + [dict(off=None), dict(pairs=-1), dict(pairs=0), dict(params=(0.0, 0, 0, 1)),
                                        dict(params=(math.inf, 0, 0, 1)), dict(params=(0.1, -0.1, 0, 1)),
                                        dict(params=(0.1, 1.1, 0, 1)), dict(params=(0.1, 0, math.nan, 1)),
                                        dict(params=(0.1, 0, 0, math.inf))])
def test_preference_refusals(L, bad):
    assert preference(L, **bad) == _abi().PR_ERR_INVALID_ARG


def test_too_many(L):
    a = _abi()
    assert policy(L, n=(1 << 26) + 1) == a.PR_ERR_UNSUPPORTED
    assert preference(L, pairs=1 << 30) == a.PR_ERR_UNSUPPORTED


def test_defaults(L):
    a = _abi()
    p, q = a.PolicyParams(), a.PreferenceParams()
    L.pr_policy_params_default(C.byref(p))
    L.pr_preference_params_default(C.byref(q))
    assert (p.clip_low, p.clip_high, p.kl_coef, p.grad_scale) == (0.2, 0.2, 0.0, 1.0)
    assert (q.beta, q.label_smoothing, q.margin, q.grad_scale) == (0.1, 0.0, 0.0, 1.0)
    L.pr_policy_params_default(None)
    L.pr_preference_params_default(None)


def test_workspace_sizes_of_the_losses(L):
    a = _abi()
    for n in (0, -3):
        assert L.pr_policy_loss_workspace(a.PR_F32, n, 1000) == 0
        assert L.pr_preference_loss_workspace(a.PR_F32, n, 1000, 0) == 0
    assert L.pr_policy_loss_workspace(a.PR_F32, 1000, 1000) <= 64 * 1000
    assert L.pr_preference_loss_workspace(a.PR_BF16, 17904, 151936, 32) <= 64 * 17904


@pytest.mark.parametrize("bad", [dict(n=-1), dict(param=None), dict(m=None), dict(v=None), dict(param=C.c_void_p(4097)),
                                 dict(m=C.c_void_p(4098)), dict(grad=C.c_void_p(4097)), dict(copy=C.c_void_p(4097)),
                                 dict(bits=16), dict(bits=8), dict(pdtype=4), dict(gdtype=-1), dict(pdtype=1, copy=P),
                                 dict(count=-1), dict(tensors=None), dict(n=1 << 60)])
def test_adamw_create_refusals(L, bad):
    a = _abi()
    x = dict(param=P, grad=P, copy=None, m=P, v=P, m_exp=None, v_exp=None, n=10)
    x.update({k: v for k, v in bad.items() if k in x})
    T = (a.AdamWTensor * 1)()
    for k, v in x.items():
        setattr(T[0], k, v)
    h = C.c_void_p(5)
    st = L.pr_adamw_create(None if "tensors" in bad else T, bad.get("count", 1), bad.get("pdtype", a.PR_F32),
                           bad.get("gdtype", a.PR_F32), bad.get("bits", 32), 0, C.byref(h))
    assert st == a.PR_ERR_INVALID_ARG and not h.value
    assert L.pr_adamw_create(T, 1, a.PR_F32, a.PR_F32, 32, 0, None) == a.PR_ERR_INVALID_ARG


def test_adamw_other_refusals(L):
    a = _abi()
    p = a.AdamWParams(0.1, 0.9, 0.999, 1e-8, 0.0, 1.0, 1)
    assert L.pr_adamw_step(None, None, C.byref(p), None) == a.PR_ERR_INVALID_ARG
    assert L.pr_adamw_moments(None, P, P, None) == a.PR_ERR_INVALID_ARG
    L.pr_adamw_destroy(None)  # ignored


def test_bindings_refuse_host_tensors():
    import torch

    import paper_2608_28726_amd as pr
    z, ids, f = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32), torch.zeros(2)
    with pytest.raises(ValueError):
        pr.policy_loss(z, ids, f, f, f, f)
    with pytest.raises(ValueError):
        pr.preference_loss(z, ids, f, f, torch.tensor([0, 1, 2], dtype=torch.int32))
    with pytest.raises(ValueError):
        pr.AdamW([f])
