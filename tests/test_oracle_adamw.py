"""The AdamW oracle against an independent implementation in float64, and the
8-bit states against their definition. CPU only."""

import numpy as np
import pytest
import torch

from oracle import adamw as oadam


def test_step_matches_an_independent_one():
    rng = np.random.default_rng(1)
    p0 = rng.normal(0, 1, 50)
    q = torch.nn.Parameter(torch.tensor(p0, dtype=torch.float64))
    opt = torch.optim.AdamW([q], lr=0.01, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    p, m, v = p0, np.zeros(50), np.zeros(50)
    for t in range(1, 6):
        g = rng.normal(0, 1, 50)
        q.grad = torch.tensor(g)
        opt.step()
        p, m, v = oadam.adamw(p, g, m, v, t, 0.01, 0.8, 0.95, 1e-6, 0.1)
        assert np.abs(p - q.detach().numpy()).max() < 1e-14


@pytest.mark.parametrize("moment", ["m", "v"])
def test_codes_bracket_their_values(moment):
    """With any random bits a value goes to one of its two neighbours, with none (0) to the lower one; a code's own
    value stays as it is; values too small for the block go to 0 (m) or to the least code (v)."""
    rng = np.random.default_rng(2)
    x = (rng.normal(0, 1, 700) * np.exp(rng.normal(0, 2, 700)) * 1e-3).astype(np.float32)
    x[5] = 0.0
    if moment == "v":
        x = x * x
    low, E = oadam.encode(x, np.zeros(700, int), moment)
    high, E2 = oadam.encode(x, np.full(700, 0xFFFFF), moment)
    assert (E == E2).all() and E.min() >= (16 if moment == "m" else 32)
    a, b = np.abs(oadam.decode(low, E, moment)), np.abs(oadam.decode(high, E, moment))
    big = np.abs(x) > np.repeat([np.abs(x[i:i + 256]).max() for i in range(0, 700, 256)], 256)[:700] * 2.0 ** -13
    mag = np.abs(x.astype(np.float64))
    assert (a[big] <= mag[big]).all() and (b[big] >= mag[big]).all() and (b[big] <= a[big] * 1.126).all()
    assert a[5] == 0 and b[5] == 0
    assert (np.sign(oadam.decode(low, E, moment))[big] == np.sign(x)[big]).all()
    again, E3 = oadam.encode(oadam.decode(low, E, moment).astype(np.float32), np.zeros(700, int), moment)
    assert (oadam.decode(again, E3, moment) == oadam.decode(low, E, moment)).all()
    tiny = np.full(256, 1e-30, np.float32)
    tiny[0] = 1.0
    k, E = oadam.encode(tiny, np.full(256, 0xFFFFF), moment)
    got = oadam.decode(k, E, moment)
    assert got[0] == 1.0 and (got[1:] == 0).all() if moment == "m" else (got[1:] > 0).all() and (got[1:] < 1e-9).all()


def test_rounding_is_right_on_average():
    """Over 4,096 steps' random bits the mean of a value's codes is the value: each is off by at most half a spacing's
    standard deviation, x / 8 / 2 / sqrt(4096) = x / 1024; five of them and a block's 256 elements give the bound."""
    x = np.linspace(1.0, 1.9, 256).astype(np.float32)
    total = np.zeros(256)
    for step in range(4096):
        bits = oadam.random_bits(256, 3, 11, step)
        k, E = oadam.encode(x, (bits & np.uint64(0xFFFFF)).astype(np.int64), "m")
        place = k.astype(np.int64) + 8 * (int(E[0]) - 15)
        total += (1 + (place % 8) / 8) * 2.0 ** (place // 8 - 127)
    assert np.abs(total / 4096 - x).max() < 5 * 1.9 / 1024


def test_random_bits_are_spread():
    """Bits of neighbouring elements, tensors and steps: each bit is set about half the time, and no two streams agree."""
    a = oadam.random_bits(1 << 14, 0, 5, 1)
    for b in (oadam.random_bits(1 << 14, 1, 5, 1), oadam.random_bits(1 << 14, 0, 5, 2), oadam.random_bits(1 << 14, 0, 6, 1),
              np.roll(a, 1)):
        same = a ^ b
        for bit in range(32):
            share = float(((same >> np.uint64(bit)) & np.uint64(1)).mean())
            assert abs(share - 0.5) < 5 * 0.5 / 128, (bit, share)


def test_nonfinite_block():
    x = np.ones(300, np.float32)
    x[7] = np.nan
    k, E = oadam.encode(x, np.zeros(300, int), "m")
    got = oadam.decode(k, E, "m")
    assert E[0] == 255 and np.isnan(got[:256]).all() and (got[256:] == 1.0).all()
