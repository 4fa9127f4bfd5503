"""Calls of more rows or requests than a launch holds are refused: a launch of 2^32 threads and more leaves the last ones
out without an error."""

import ctypes as C

import pytest

from tests.helpers import ensure_built

P = C.c_void_p(4096)


@pytest.fixture(scope="module")
def L():
    return ensure_built()


def test_rows_beyond_a_launch_are_refused(L):
    from paper_2608_28726_amd import _abi as a
    out = a.TokenFeatures(*[P] * len(a.FEATURE_FIELDS))
    for n, top_p in ((1 << 24, None), ((1 << 26), None), (1 << 23, P), ((1 << 23) + 5, P)):
        args = (P, a.PR_F32, n, 8, 8, P, P, top_p)
        assert L.pr_token_features_ws(*args, C.byref(out), None, 0, None) == a.PR_ERR_UNSUPPORTED, (n, top_p)
        assert L.pr_token_features_noalloc(*args, C.byref(out), None) == a.PR_ERR_UNSUPPORTED, (n, top_p)
        assert L.pr_feature_sequence(*args, P, 1, 20, P, None, None) == a.PR_ERR_UNSUPPORTED, (n, top_p)
    for n in (1 << 24, (1 << 25) + 3):
        assert L.pr_sample_features(P, a.PR_BF16, n, 8, 8, P, 1, 0, P, None, None, 0, 20, None, None) == a.PR_ERR_UNSUPPORTED


def test_requests_beyond_a_launch_are_refused(L):
    from paper_2608_28726_amd import _abi as a
    out, agg = a.TokenFeatures(*[P] * len(a.FEATURE_FIELDS)), a.RequestAgg(P, P, P, P, P)
    assert L.pr_request_aggregate(C.byref(out), P, 1 << 24, None, C.byref(agg), None) == a.PR_ERR_UNSUPPORTED


@pytest.mark.gpu
@pytest.mark.parametrize("top_p", [None, 0.5])
def test_as_many_rows_as_a_launch_holds(top_p):
    import torch

    import paper_2608_28726_amd as pr
    from tests.gpu_common import require_gpu
    require_gpu()
    n = (1 << (24 if top_p is None else 23)) - 1
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    z = torch.empty(n, 3, device="cuda").normal_(generator=g)
    T = torch.ones(n, device="cuda")
    P_row = None if top_p is None else torch.full((n,), top_p, device="cuda")
    f = pr.token_features(z, torch.zeros(n, dtype=torch.int32, device="cuda"), T, P_row)
    assert torch.equal(f["argmax"].long(), z.argmax(1)) and (f["flags"] & 7 == 0).all()
    part = slice(n - 1000, n)
    if top_p is None:
        lp = torch.log_softmax(z[part].double(), 1)[:, 0]
        assert ((f["logprob"][part].double() - lp).abs() <= 1e-5 + 1e-4 * lp.abs()).all()
        offsets = torch.arange(n + 1, dtype=torch.int32, device="cuda")
        agg = pr.request_aggregate(f, offsets)
        torch.cuda.synchronize()
        assert torch.equal(agg["score"], f["maxprob"])  # a request a row
        ids, _, _ = pr.sample_features(z, T, 1, features=False)
        assert ((ids >= 0) & (ids < 3)).all()
    torch.cuda.synchronize()
    with pytest.raises(pr.ProuterError):
        pr.token_features(torch.zeros(n + 1, 2, device="cuda"), torch.zeros(n + 1, dtype=torch.int32, device="cuda"),
                          torch.ones(n + 1, device="cuda"), None if top_p is None else torch.ones(n + 1, device="cuda"))
