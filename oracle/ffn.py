"""4-bit weights and the gated feed-forward projection, float64.

The format (OCP microscaling FP4): a code's bit 3 is the sign, bits 2-1 an
exponent field of bias 1, bit 0 the mantissa; 32 columns of a row share a power of
two.  A group takes the least exponent in [-125, 125] at which its largest
magnitude is 6 or below, each value the nearest code, ties to the even one.  A
group with a value that is not finite has byte 255, which makes it NaN.
"""
from __future__ import annotations

import numpy as np

from . import linear as ol

GROUP = 32


def code_value(code: int) -> float:
    field, half = (code >> 1) & 3, code & 1
    size = half * 0.5 if field == 0 else (1 + half * 0.5) * 2.0 ** (field - 1)
    return -size if code & 8 else size


VALUES = np.array([code_value(c) for c in range(16)])


def unpack(codes) -> np.ndarray:
    """uint8 [n][k / 2] -> one code a column."""
    c = np.asarray(codes, dtype=np.uint8)
    return np.stack([c & 15, c >> 4], -1).reshape(c.shape[0], -1)


def values(codes, exps) -> np.ndarray:
    """What 4-bit weights stand for, float64 [n][k]."""
    e = np.asarray(exps, dtype=np.float64)
    scale = np.where(e == 255, np.nan, 2.0 ** (e - 127))
    return VALUES[unpack(codes)] * np.repeat(scale, GROUP, axis=1)


def quantize(w):
    """float64 [n][k] -> (one code a column, exponent bytes), group by group."""
    w = np.asarray(w, dtype=np.float64)
    n, k = w.shape
    codes = np.zeros((n, k), dtype=np.uint8)
    exps = np.zeros((n, k // GROUP), dtype=np.uint8)
    for i in range(n):
        for g in range(k // GROUP):
            v = w[i, g * GROUP:(g + 1) * GROUP]
            if not np.isfinite(v).all():
                exps[i, g] = 255
                continue
            e = -125
            while e < 125 and np.abs(v).max() > 6.0 * 2.0 ** e:
                e += 1
            exps[i, g] = e + 127
            size = np.abs(v) / 2.0 ** e
            # nearest magnitude; of two as near the even code
            far = np.abs(size[:, None] - VALUES[None, :8])
            nearest = [np.flatnonzero(row == row.min()) for row in far]
            pick = np.array([c[0] if len(c) == 1 or c[0] % 2 == 0 else c[1] for c in nearest])
            codes[i, g * GROUP:(g + 1) * GROUP] = pick + 8 * np.signbit(v)
    return codes, exps


def activate(g, act: str) -> np.ndarray:
    g = np.asarray(g, dtype=np.float64)
    y = g if act == "silu" else 2.0 * np.sqrt(2.0 / np.pi) * (g + 0.044715 * g ** 3)
    with np.errstate(over="ignore"):
        return g / (1.0 + np.exp(-y))


def gated_linear(x, gate, up, act: str = "silu") -> np.ndarray:
    """x: float64 [m][k]; gate, up: float64 [n][k]."""
    return activate(ol.linear(x, gate), act) * ol.linear(x, up)
