"""GPU: projections whose first choice of a form would be 2^32 threads take another one."""
import math

import pytest
import torch

import _projections as pj
from oracle import ffn as of
from paper_2609_38386_amd import dlfp as D
from paper_2609_38386_amd import runtime as rt

pytestmark = pytest.mark.gpu


def test_features_past_one_form():
    """One token of 2^29 features, and of 2^28 gates and ups: weights 0 but for a few rows at the
    ends and between (36 GB in all)."""
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev)
    gen.manual_seed(8)
    n, k, rows = 1 << 29, 128, 48
    codes = torch.zeros((n, k // 2), dtype=torch.uint8, device=dev)
    exps = torch.full((n, k // 32), 120, dtype=torch.uint8, device=dev)
    starts = [0, n // 4 + 16, n // 2 - rows, n // 2, 3 * n // 4, n - rows]
    for at in starts:
        codes[at:at + rows], exps[at:at + rows] = pj.random_codes(gen, rows, k, device=dev)

    def values(at):
        return of.values(codes[at:at + rows].cpu().numpy(), exps[at:at + rows].cpu().numpy())

    x = torch.empty((1, k), dtype=torch.float32, device=dev).normal_(generator=gen).to(torch.bfloat16)
    out = torch.full((1, n), math.nan, dtype=torch.float32, device=dev)
    rt.linear(x, rt.Weights4.of(codes, exps), out)
    for at in starts:
        pj.check(out[:, at:at + rows], *pj.linear(pj.f64(x), values(at), torch.float32))
    zeros = torch.ones((n,), dtype=torch.bool, device=dev)
    for at in starts:
        zeros[at:at + rows] = False
    assert not (out[0] * zeros).any()

    half = n // 2
    gate, up = (rt.Weights4.of(codes[i * half:(i + 1) * half], exps[i * half:(i + 1) * half])
                for i in range(2))
    out = out[:, :half].fill_(math.nan)
    rt.gated_linear(x, gate, up, out)
    assert not out.isnan().any()
    for at in (0, half - rows):       # rows of the gate; the up's begin at n / 2
        if at == 0:
            want = pj.gated(pj.f64(x), values(0), values(half), "silu", torch.float32)
        else:
            want = pj.gated(pj.f64(x), values(half - rows), values(n - rows), "silu", torch.float32)
        pj.check(out[:, at:at + rows], *want)
    assert D.dlfp_projection_form_of(D.LINEAR_W4, 1, n, k, 0).variant >= 0
