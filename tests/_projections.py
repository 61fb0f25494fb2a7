"""Inputs and bounds of the projection tests.

Bounds.  An output is a sum over k of exact products in fp32, in an unknown order:
k / 16 matrix instructions of 16 columns at least, each of which may round twice (its own
sum and the addition to the accumulator) or drop bits below 2^-23 of the larger, and up to
32 partial sums.  Every partial sum is at most S = sum |x| |w|, so a sum is off by at most
(k / 16 + 32) 2^-23 S.  With a gate g off by dg and an up u off by du, act(g) u is off by at
most 1.13 |u| dg + (|act(g)| + 1.13 dg) du (no slope of either activation is over 1.13),
and the activation's own arithmetic by (4 |y| + 10) 2^-24 of it, y the power's argument
(four roundings of y, which count |y| times in e^y, and ten of the rest).  The last rounding
to bf16 adds 2^-8 of the value.
"""
import numpy as np
import torch

from oracle import attention as oa
from oracle import ffn as of
from oracle import linear as ol

SLOPE = 1.13


def f64(t):
    if t.dtype == torch.bfloat16:
        return oa.bf16_bits_to_float64_tensor(t.contiguous().view(torch.int16).cpu()).numpy()
    return t.double().cpu().numpy()


def sum_bound(x, w):
    k = x.shape[1]
    return (k / 16 + 32) * 2.0 ** -23 * ol.linear(np.abs(x), np.abs(w))


def rounded(want, bound, dtype):
    return bound + (2.0 ** -8 * (np.abs(want) + bound) if dtype == torch.bfloat16 else 0.0)


def linear(x, w, dtype):
    """(exact result, bound)."""
    want = ol.linear(x, w)
    return want, rounded(want, sum_bound(x, w), dtype)


def gated(x, gate, up, act, dtype):
    g, u = ol.linear(x, gate), ol.linear(x, up)
    dg, du = sum_bound(x, gate), sum_bound(x, up)
    a = of.activate(g, act)
    want = a * u
    y = np.abs(g) if act == "silu" else np.abs(1.6 * (g + 0.044715 * g ** 3))
    own = np.abs(want) * (4 * y + 10) * 2.0 ** -24
    bound = SLOPE * np.abs(u) * dg + (np.abs(a) + SLOPE * dg) * du + own
    return want, rounded(want, bound, dtype)


def random_codes(gen, n, k, lo=118, hi=124, device="cpu"):
    """Codes of every kind, exponents a few apart."""
    codes = torch.randint(0, 256, (n, k // 2), generator=gen, device=device, dtype=torch.uint8)
    exps = torch.randint(lo, hi, (n, k // 32), generator=gen, device=device, dtype=torch.uint8)
    return codes, exps


def check(got, want, bound):
    got = f64(got)
    off = np.abs(got - want)
    assert np.isfinite(got).all()
    assert (off <= bound).all(), (off.max(), float((off / np.maximum(bound, 1e-300)).max()))
