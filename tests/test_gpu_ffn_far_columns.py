"""GPU: rows of 2^22 columns and more, up to the longest that a 32-bit size can name."""
import math

import pytest
import torch

import _projections as pj
from oracle import ffn as of
from paper_2609_38386_amd import runtime as rt

pytestmark = pytest.mark.gpu


@pytest.fixture
def gen():
    g = torch.Generator(device="cuda:0")
    g.manual_seed(12)
    return g


@pytest.mark.parametrize("m", [1, 40])
def test_rows_of_four_million_columns(gen, m):
    """Every call with K past the 32-bit offsets, gate and up not 0 in three pieces of a row."""
    dev, n, k = torch.device("cuda:0"), 48, (1 << 22) + 64
    pieces = [slice(0, 64), slice(1 << 21, (1 << 21) + 256), slice(k - 192, k)]
    x = torch.empty((m, k), dtype=torch.bfloat16, device=dev).normal_(generator=gen)
    dense = [torch.zeros((n, k), dtype=torch.bfloat16, device=dev) for _ in range(2)]
    for d in dense:
        for p in pieces:
            d[:, p] = torch.empty((n, p.stop - p.start), device=dev).normal_(generator=gen) * 0.05
    four = [rt.Weights4.from_bf16(d) for d in dense]
    some = lambda t: torch.cat([t[:, p] for p in pieces], 1)  # noqa: E731
    x64 = pj.f64(some(x))
    out = torch.empty((m, n), dtype=torch.float32, device=dev)
    rt.gated_linear(x, *dense, out)
    pj.check(out, *pj.gated(x64, pj.f64(some(dense[0])), pj.f64(some(dense[1])), "silu",
                            torch.float32))
    for w, d in zip(four, dense):
        w.dequantize(d)
    values = [pj.f64(some(d)) for d in dense]
    rt.linear(x, four[0], out)
    pj.check(out, *pj.linear(x64, values[0], torch.float32))
    rt.gated_linear(x, *four, out, "gelu")
    pj.check(out, *pj.gated(x64, *values, "gelu", torch.float32))


def test_the_longest_rows(gen):
    """2^31 - 64 columns (22 GB): the step behind the last one is past 31 bits."""
    dev, n, k = torch.device("cuda:0"), 16, (1 << 31) - 64
    codes = torch.zeros((n, k // 2), dtype=torch.uint8, device=dev)
    exps = torch.full((n, k // 32), 120, dtype=torch.uint8, device=dev)
    x = torch.zeros((1, k), dtype=torch.bfloat16, device=dev)
    # [first column, columns): both ends and a piece past 2^30.
    pieces = [(0, 128), ((1 << 30) + 96 * 32, 64), (k - 1984, 1984)]
    xs, values = [], []
    for at, count in pieces:
        c, e = pj.random_codes(gen, n, count, device=dev)
        codes[:, at // 2:(at + count) // 2], exps[:, at // 32:(at + count) // 32] = c, e
        x[:, at:at + count] = torch.empty((1, count), device=dev).normal_(generator=gen)
        xs.append(x[:, at:at + count])
        values.append(torch.from_numpy(of.values(c.cpu().numpy(), e.cpu().numpy())))
    out = torch.full((1, n), math.nan, dtype=torch.float32, device=dev)
    torch.cuda.synchronize()
    rt.linear(x, rt.Weights4.of(codes, exps), out)
    torch.cuda.synchronize()
    pj.check(out, *pj.linear(pj.f64(torch.cat(xs, 1)), torch.cat(values, 1).numpy(),
                             torch.float32))
