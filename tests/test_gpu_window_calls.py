"""GPU: calls of windowed and 8-bit attention at the ends of what they take."""
import math

import numpy as np
import pytest
import torch

from _paged_mixes import bf16
from paper_2609_38386_amd import dlfp as D
from paper_2609_38386_amd import runtime as rt

pytestmark = pytest.mark.gpu
SCALE = 1.0 / math.sqrt(128)
SWAP = [(t & 3) | ((t & 4) << 1) | ((t & 8) >> 1) for t in range(16)]
BF16, FP32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available()
    D.lib()
    return torch.device("cuda:0")


@pytest.fixture(scope="module")
def ws(dev):
    return rt.Workspace(dev, 16 << 20)


def test_context_past_a_million_keys(dev, ws):
    """A decoder of 1050001 keys, whose pages are 40 blocks of the pool over and over, so
    that the oracle is a sum over 640 keys with their counts.

    Bounds as in _paged_mixes.Mix.check, with two roundings of the sums in place of its
    one for 16 keys: a wavefront's quarter of a unit of 4096 keys is 64 products, and
    257 partial results follow."""
    n, blocks, rng = 1050001, 40, np.random.default_rng(3)
    table = rng.integers(0, blocks, size=(1, -(-n // 16))).astype(np.int32)
    k, v = (bf16(rng.normal(size=(blocks, 1, 16, 128))) for _ in "kv")
    q = bf16(rng.normal(size=(1, 2, 128)))
    pool = rt.KVPool.of(k.to(dev), v[:, :, SWAP].transpose(2, 3).contiguous().to(dev))
    count = np.repeat(np.bincount(table[0, :-1], minlength=blocks), 16).astype(np.float64)
    last = n - 16 * (table.size - 1)
    count[16 * table[0, -1]:16 * table[0, -1] + last] += 1
    assert count.sum() == n
    kk, vv = (x.double().numpy().reshape(-1, 128) for x in (k, v))
    score = SCALE * (q[0].double().numpy() @ kk.T)
    w = count * np.exp(score - score.max(1, keepdims=True))
    w /= w.sum(1, keepdims=True)
    want = w @ vv
    spread = np.stack([(w[h][:, None] * np.abs(vv - want[h])).sum(0) for h in range(2)])
    magnitude = SCALE * (np.abs(q[0].double().numpy()) @ np.abs(kk).T).max()
    batch = rt.WindowBatch(D.make_dims(2, 1), [1], [n], table, blocks, dev)
    for dtype, half, term in ((BF16, 2.0 ** -8, 2.0 ** -15), (FP32, 2.0 ** -24, 2.0 ** -21)):
        out = torch.full((1, 2, 128), float("nan"), dtype=dtype, device=dev)
        batch.attention(pool, q.to(dev), SCALE, out, ws)
        d = 128 * 2.0 ** -24 * magnitude + 2.0 ** -18 + term
        tol = (half * np.abs(want) + 2 * d / (1 - d) * spread +
               (64 + 257 + 16) * 2.0 ** -24 * (w @ np.abs(vv)))
        err = np.abs(out[0].double().cpu().numpy() - want)
        assert (err <= tol).all(), float((err / tol).max())
    assert D.dlfp_workspace_error(ws.buf) == 0
