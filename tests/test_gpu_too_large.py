"""Sizes beyond 32 bits are refused: they are never taken for their lower 32 bits."""

import pytest
import torch

import paper_2608_28726_amd as pr
from tests.gpu_common import require_gpu

pytestmark = pytest.mark.gpu

OVER = 2 ** 32 + 5  # 5 in 32 bits


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()
    yield
    torch.cuda.empty_cache()


def test_a_vocabulary_beyond_32_bits():
    z = torch.empty(1, OVER, dtype=torch.bfloat16, device="cuda")
    f, i = torch.ones(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    state = pr.StreamState(1, 4)
    for call in (lambda: pr.top_logits(z, 2), lambda: pr.beam_select(z, f[None]),
                 lambda: pr.distill_loss(z, i[None], f[None], 1.0, f, grad=False),
                 lambda: pr.policy_loss(z, i, 1.0, f, f, f, grad=False),
                 lambda: pr.preference_loss(z, i, 1.0, f, torch.zeros(3, dtype=torch.int32, device="cuda"), grad=False),
                 lambda: pr.token_features(z, i, f), lambda: pr.sample_features(z, f, 1), lambda: state.step(z, i, i, f)):
        with pytest.raises(ValueError, match="2\\^31"):
            call()
    state.close()


def test_more_requests_than_32_bits_count():
    parent = torch.empty(OVER, 1, dtype=torch.int32, device="cuda")
    slots = torch.empty(OVER, 1, dtype=torch.int32, device="cuda")
    state = pr.StreamState(8, 4)
    with pytest.raises(ValueError, match="2\\^31"):
        pr.beam_reorder([], parent)
    with pytest.raises(ValueError, match="2\\^31"):
        state.reorder(slots, parent)
    state.close()
    z = torch.empty(OVER, 2, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError, match="2\\^31"):
        pr.beam_select(z, torch.empty(OVER, 1, device="cuda"))
