"""GPU: the gated projection's activation where the gate is far below 0 and all of its value is in
the power: e^-y from 2^80 to past fp32's largest number.

Gates and ups are one exact product each (a column of ones), so that what is off is the activation's
arithmetic.  In half steps (2^-24 of the value): SiLU's power 2 and the rounding that puts its
product's error back 1, 1 + e 1, the reciprocal 2, two products 2: 8.  GELU's y has seven roundings
(two constants, five operations), which count |y| times in e^-y.  An activation below 2^-126 is
rounded to a multiple of 2^-149, at most that much off, which counts |u| times; so does an output.
"""
import numpy as np
import pytest
import torch

import _projections as pj
from oracle import ffn as of
from paper_2609_38386_amd import dlfp as D
from paper_2609_38386_amd import runtime as rt

pytestmark = pytest.mark.gpu

EACH = 256


def _gates(act):
    lo, hi = (-104.0, -56.0) if act == "silu" else (-11.0, -8.5)
    return torch.linspace(lo, hi, EACH).to(torch.bfloat16)


def _bound(g, u, act, want):
    y = 0.0 if act == "silu" else 1.6 * (np.abs(g) + 0.044715 * np.abs(g) ** 3)
    return np.abs(want) * (7 * y + 8 * 1.0001) * 2.0 ** -24 + (np.abs(u) + 1) * 2.0 ** -149


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("form", ["few", "split", "tiles", "far"])
def test_gates_far_below_zero(act, form):
    dev = torch.device("cuda:0")
    k = 16384 if form == "split" else 64
    m = 300 if form == "tiles" else 1 if form == "few" else 40
    ups = (1.0, 2.0 ** 40, 2.0 ** 90)
    n = EACH * len(ups)
    gate, up = (torch.zeros((n, k), dtype=torch.bfloat16, device=dev) for _ in range(2))
    gate[:, 0] = _gates(act).repeat(len(ups)).to(dev)
    up[:, 1] = torch.tensor(ups).repeat_interleave(EACH).to(torch.bfloat16).to(dev)
    ld = (1 << 22) + 8 if form == "far" else k
    x = torch.zeros(((m - 1) * ld + k,), dtype=torch.bfloat16, device=dev).as_strided((m, k), (ld, 1))
    x[:, :2] = 1.0
    out = torch.full((m, n), 7.0, dtype=torch.float32, device=dev)
    if form == "split":
        assert D.dlfp_projection_workspace(D.GATED_LINEAR_BF16, m, n, k) > 0
    rt.gated_linear(x, gate, up, out, act)
    g, u = pj.f64(gate[:, 0]), pj.f64(up[:, 1])
    want = of.activate(g, act) * u
    assert np.abs(want).min() < 2.0 ** -140 and np.abs(want).max() > 2.0 ** 10
    pj.check(out, want[None], _bound(g, u, act, want)[None])


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gates_without_end(act):
    """The largest finite gates: 0 below, the gate itself above; an infinite one above too."""
    dev = torch.device("cuda:0")
    most = float(torch.finfo(torch.bfloat16).max)
    values = [-most, -1e30, -1e13, -3000.0, -200.0, 200.0, 1e13, most]
    gate, up = (torch.zeros((16, 64), dtype=torch.bfloat16, device=dev) for _ in range(2))
    gate[:len(values), 0] = torch.tensor(values).to(torch.bfloat16).to(dev)
    up[:, 1] = 0.5
    x = torch.zeros((1, 64), dtype=torch.bfloat16, device=dev)
    x[0, :2] = 1.0
    out = torch.empty((1, 16), dtype=torch.float32, device=dev)
    rt.gated_linear(x, gate, up, out, act)
    got, g = pj.f64(out)[0], pj.f64(gate[:, 0])
    assert not got[:5].any()
    assert np.array_equal(got[5:len(values)], 0.5 * g[5:len(values)])
