"""Oracle: the AdamW step in float64, and the 8-bit states bit by bit.

TEST INFRASTRUCTURE ONLY -- see the package docstring. Shares no code with
the HIP library.

Reading:

R27  8-bit states. 256 elements of a tensor share an exponent byte E. With
     base = 8 (E - 15) for m and 8 (E - 31) for v, code k > 0 stands for the
     float32 whose bits are (k + base) << 20, code 0 for 0; m has a sign bit
     besides. On writing, E is the exponent of the block's largest magnitude
     with its 20 low bits rounded up, at least 16 (m) or 32 (v); a value is
     its bits' upper part after 20 random bits have been added, minus the
     base; results below 1 are 0 for m and 1 for a positive v.
     E = 255 marks a block that holds a NaN, an infinity or a magnitude above
     15/8 2^127.
"""

from __future__ import annotations

import math

import numpy as np

BLOCK = 256


def adamw(p, g, m, v, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.01, grad_scale=1.0):
    """One step in float64: p', m', v'."""
    p, g, m, v = (np.asarray(x, dtype=np.float64) for x in (p, g, m, v))
    g = g * grad_scale
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    mhat, vhat = m / (1 - beta1 ** step), v / (1 - beta2 ** step)
    return p - lr * weight_decay * p - lr * mhat / (np.sqrt(vhat) + eps), m, v


def random_bits(n: int, tensor: int, seed: int, step: int) -> np.ndarray:
    """The 32 random bits of each element of a tensor."""
    x = (seed + step * 0x9E3779B97F4A7C15) % 2 ** 64
    x = (x ^ (x >> 30)) * 0xBF58476D1CE4E5B9 % 2 ** 64
    x = (x ^ (x >> 27)) * 0x94D049BB133111EB % 2 ** 64
    key = (x ^ (x >> 31)) >> 32

    def mix(a):
        a = a * np.uint64(0x9E3779B9) % np.uint64(2 ** 32)
        a = a ^ (a >> np.uint64(15))
        a = a * np.uint64(0x6A09E667) % np.uint64(2 ** 32)
        return a ^ (a >> np.uint64(13))

    k = mix(np.array([(tensor + 1 + key) % 2 ** 32], dtype=np.uint64))
    return mix((np.arange(n, dtype=np.uint64) + k) % np.uint64(2 ** 32))


def encode(x, random, moment: str):
    """Codes (uint8) and block exponents (uint8) of float32 values."""
    x = np.asarray(x, dtype=np.float32)
    top = 15 if moment == "m" else 31
    mag = (x.view(np.uint32) & np.uint32(0x7FFFFFFF)).astype(np.int64)
    n_blocks = -(-len(x) // BLOCK)
    codes, exps = np.zeros(len(x), np.uint8), np.zeros(n_blocks, np.uint8)
    for b in range(n_blocks):
        part = slice(b * BLOCK, min(len(x), (b + 1) * BLOCK))
        E = int(min(255, max(top + 1, (mag[part].max() + 0xFFFFF) >> 23)))
        k = ((mag[part] + np.asarray(random[part], dtype=np.int64)) >> 20) - 8 * (E - top)
        k = np.where(mag[part] > 0, np.maximum(k, 0 if moment == "m" else 1), 0) % (8 * (top + 1))
        if moment == "m":
            k = k + np.where(x[part] < 0, 128, 0)
        codes[part], exps[b] = k, E
    return codes, exps


def decode(codes, exps, moment: str) -> np.ndarray:
    """Values (float64) of codes under their blocks' exponents."""
    top = 15 if moment == "m" else 31
    out = np.zeros(len(codes))
    for i, c in enumerate(np.asarray(codes).tolist()):
        E = int(exps[i // BLOCK])
        k, sign = (c & 127, -1.0 if c & 128 else 1.0) if moment == "m" else (c, 1.0)
        place = k + 8 * (E - top)  # 8 per octave, from 2^-127
        if E == 255:
            out[i] = math.nan
        elif k:
            out[i] = sign * math.ldexp(1.0 + (place % 8) / 8.0, place // 8 - 127)
    return out
