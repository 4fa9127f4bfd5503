"""The features' oracle on rows far from zero, where what the logits have in common must not reach the log-prob (CPU
only)."""

import numpy as np
import pytest

import oracle


@pytest.mark.parametrize("shift", [0.0, 1e10, -1e25])
@pytest.mark.parametrize("P", [None, 0.9])
def test_log_prob_of_equal_logits(shift, P):
    V = 400
    f = oracle.token_features(np.full(V, shift, np.float32), "f32", 7, 1.0, P)
    kept = V if P is None else f["cutoff"]
    assert f["flags"] == 0 and abs(f["logprob"] + np.log(kept)) <= 1e-12 and abs(f["entropy"] - np.log(kept)) <= 1e-12
