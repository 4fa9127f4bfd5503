"""The post-training example: losses, gradients and optimizer working together raise what the answers earn."""

import math

import pytest

from paper_2608_28726_amd.post_train import post_train
from tests.gpu_common import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("method", ["policy", "preference"])
@pytest.mark.parametrize("state_bits", [8, 32])
def test_reward_rises(method, state_bits):
    """A quarter of the vocabulary earns a point: the mean starts near 0.25 (standard deviation of 512 draws 0.02) and
    ends well above."""
    out = post_train(method, steps=60, state_bits=state_bits)
    print(method, state_bits, out["reward"][0], out["reward_after"], flush=True)
    assert all(math.isfinite(v) for v in out["loss"])
    assert out["reward"][0] < 0.35 and out["reward_after"] > 0.5
    if method == "preference":  # each pair starts where the reference is
        assert abs(out["loss"][0] - math.log(2.0)) < 1e-3


def test_unknown_method():
    with pytest.raises(ValueError):
        post_train("reward", steps=1)
