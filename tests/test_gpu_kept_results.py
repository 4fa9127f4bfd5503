"""Results that a program keeps hold the memory of the call's results, not of its scratch."""

import pytest
import torch

import paper_2608_28726_amd as pr
from paper_2608_28726_amd import _abi
from tests.gpu_common import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def rows(n, V, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(n + V)
    return torch.empty(n, V, dtype=torch.float32, device="cuda").normal_(generator=g).to(dtype)


def held(out):
    """Bytes of all storages behind the outputs, each once, beside the bytes of the outputs."""
    tensors = list(out.values())
    behind = {x.untyped_storage().data_ptr(): x.untyped_storage().nbytes() for x in tensors}
    return sum(behind.values()), sum(x.numel() * x.element_size() for x in tensors)


# Rows in parts and whole ones.
@pytest.mark.parametrize("n,V,k,dtype", [(17, 151936, 64, torch.bfloat16), (17, 50257, 256, torch.bfloat16),
                                         (600, 2000, 8, torch.float32)])
def test_top_logits_and_the_losses(n, V, k, dtype):
    z = rows(n, V, dtype)
    f, w = torch.zeros(n, device="cuda"), torch.full((n,), 1.0 / n, device="cuda")
    ids = torch.arange(n, dtype=torch.int32, device="cuda")
    offsets = torch.arange(0, 2 * (n // 2) + 1, n // 2, dtype=torch.int32, device="cuda")
    top = pr.top_logits(z, k)
    even = 2 * (n // 2)
    for name, out in (("top", top), ("distill", pr.distill_loss(z, top["ids"], top["logprob"], 1.0, w)),
                      ("policy", pr.policy_loss(z, ids, 1.0, w, w, f)),
                      ("preference", pr.preference_loss(z[:even], ids[:even], 1.0, w[:even], offsets, f[:even]))):
        have, need = held(out)
        assert have == need, (name, have, need)
        if "loss" in out:  # the scalar that a training loop keeps: beside it a few floats a row
            assert out["loss"].untyped_storage().nbytes() <= 16 * n + 4, name


@pytest.mark.parametrize("n_req,B,V,k,dtype", [(1, 4, 32000, 4, torch.float32), (8, 16, 20000, 16, torch.bfloat16)])
def test_beam_select(n_req, B, V, k, dtype):
    z, scores = rows(n_req * B, V, dtype), torch.zeros(n_req, B, device="cuda")
    need = _abi.lib().pr_beam_select_workspace(_abi.PR_F32 if dtype == torch.float32 else _abi.PR_BF16, n_req, B, V, k)
    assert need > 8 * n_req * k
    out = pr.beam_select(z, scores, k=k)
    have, need = held(out)
    assert have == need
    assert out["scores"].untyped_storage().nbytes() == 8 * n_req * k  # with the log-probs
