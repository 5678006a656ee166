"""CPU oracle of activations kept in 8 bits.  TEST INFRASTRUCTURE ONLY.

A group of 128 values of a row (the last may be shorter) has the smallest bf16 scale s >= 2^-100 with 127 s >= max |x|; a
value's code is the whole number next to the fp32 quotient x / s, ties to even.  A group with a value that is not finite or
2^127 or larger has codes 0 and scale NaN.  Scales are found here by trying: the bf16 numbers around max |x| / 127 in exact
(float64) arithmetic.  Pinned by tests/test_step_pins.py."""
from __future__ import annotations

import numpy as np

GROUP = 128


def _bf16_at_least(v):
    """The smallest bf16 number >= v (v >= 0, float64)."""
    bits = np.asarray(v, dtype=np.float64).astype(np.float32).view(np.uint32) & np.uint32(0xFFFF0000)
    s = bits.view(np.float32).astype(np.float64)
    while np.any(s < v):
        bits = np.where(s < v, bits + np.uint32(0x10000), bits).astype(np.uint32)
        s = bits.view(np.float32).astype(np.float64)
    return s


def pack(X):
    """(codes int8 [T, d], scales float32 [T, groups])"""
    X = np.asarray(X, dtype=np.float32)
    T, d = X.shape
    G = (d + GROUP - 1) // GROUP
    codes, scales = np.zeros((T, d), dtype=np.int8), np.zeros((T, G), dtype=np.float32)
    for g in range(G):
        x = X[:, g * GROUP:(g + 1) * GROUP]
        top = np.abs(x.astype(np.float64)).max(axis=1)
        bad = ~(top < 2.0 ** 127)
        s = np.maximum(_bf16_at_least(np.where(bad, 0.0, top) / 127.0), 2.0 ** -100)
        q = np.rint((np.where(bad[:, None], 0, x).astype(np.float32) / s[:, None].astype(np.float32)).astype(np.float32))
        codes[:, g * GROUP:(g + 1) * GROUP] = q.astype(np.int8)
        scales[:, g] = np.where(bad, np.float32("nan"), s.astype(np.float32))
    return codes, scales


def unpack(codes, scales):
    """Values as float64, before their rounding to the tensor's type."""
    T, d = codes.shape
    return codes.astype(np.float64) * np.repeat(scales.astype(np.float64), GROUP, axis=1)[:, :d]
