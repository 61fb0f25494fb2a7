"""GPU: attention with a window and sinks over bf16 and 8-bit pages against the oracle.

Bounds are derived in _paged_mixes.Mix.check.  Whatever no row of a sequence sees
is NaN in every cache, and outputs are NaN before a launch.
"""
import math

import numpy as np
import pytest
import torch

from _paged_mixes import Mix
from paper_2609_38386_amd import dlfp as D
from paper_2609_38386_amd import runtime as rt

pytestmark = pytest.mark.gpu
SCALE = 1.0 / math.sqrt(128)
BF16, FP32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available()
    D.lib()
    return torch.device("cuda:0")


@pytest.fixture(scope="module")
def ws(dev):
    return rt.Workspace(dev, 16 << 20)


# q_len, kv_len, window, sinks
DECODE = [
    ([1], [1], None, 0), ([1, 1, 1, 1], [1, 2, 15, 16], 1, 0), ([1, 1, 1], [17, 63, 64], 5, 3),
    ([1, 1, 1], [65, 129, 700], None, 0), ([1, 1, 1], [300, 301, 302], 64, 17),
    ([1, 1], [1000, 1015], 1, 1), ([1, 1, 1], [800, 40, 1111], 257, 130),
]
PROMPT = [
    ([2], [2], None, 0), ([40], [40], 7, 2), ([17, 130], [17, 140], None, 0),
    ([65], [300], 33, 5), ([129], [700], 200, 64), ([300], [333], 1, 0), ([300], [333], 3, 31),
    ([20, 3, 64], [500, 3, 64], 128, 20),
]
MIXED = [
    ([40, 1, 1, 9], [90, 1, 200, 333], None, 0), ([130, 1, 1, 1], [400, 65, 600, 31], 100, 4),
    ([16, 1], [16, 16], 2, 1),
]


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (4, 2), (8, 2), (16, 2)])
@pytest.mark.parametrize("case", range(len(DECODE)))
def test_decode(dev, ws, case, hq, hkv, kv8):
    m = Mix(dev, hq, hkv, *DECODE[case], kv8, seed=case)
    for dtype in (BF16, FP32):
        for tn in (None, D.dlfp_tuning(64), D.dlfp_tuning(16)):
            m.check(m.run(ws, dtype, SCALE, tn), SCALE)
    assert D.dlfp_workspace_error(ws.buf) == 0


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("hq,hkv", [(2, 2), (4, 2), (8, 2), (16, 2)])
@pytest.mark.parametrize("case", range(len(PROMPT)))
def test_prompts(dev, ws, case, hq, hkv, kv8):
    m = Mix(dev, hq, hkv, *PROMPT[case], kv8, seed=case)
    for dtype, tn in ((BF16, None), (FP32, None), (BF16, D.dlfp_tuning(0, 64)),
                      (FP32, D.dlfp_tuning(0, 128, 0, 3))):
        m.check(m.run(ws, dtype, SCALE, tn), SCALE)
    assert D.dlfp_workspace_error(ws.buf) == 0


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("case", range(len(MIXED)))
def test_mixed(dev, ws, case, kv8):
    m = Mix(dev, 8, 2, *MIXED[case], kv8, seed=case)
    for dtype in (BF16, FP32):
        for tn in (None, D.dlfp_tuning(32, 64), D.dlfp_tuning(0, 0, 0, 1, 1)):
            m.check(m.run(ws, dtype, SCALE, tn), SCALE)
    assert D.dlfp_workspace_error(ws.buf) == 0


# Decode units of a wavefront each: many short ones, alone and beside a prompt, whole
# and split, in numbers that leave the last workgroup with one, two and three.
SHORT = [
    (8, 1, [1] * 37 + [400], [1 + 5 * i % 6 for i in range(37)] + [1200], None, 0, None),
    (16, 2, [1] * 61 + [800], [1 + 37 * i % 200 for i in range(61)] + [2200], None, 0, 64),
    (4, 2, [800] + [1] * 43, [2200] + [3 + 37 * i % 190 for i in range(43)], 150, 20, 64),
    (16, 2, [1] * 389, [1 + 31 * i % 97 for i in range(389)], None, 0, 64),
    (4, 2, [1] * 391, [1 + 31 * i % 211 for i in range(391)], 90, 20, 64),
]


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("case", range(len(SHORT)))
def test_short_decoders(dev, ws, case, kv8):
    hq, hkv, q_len, kv_len, window, sinks, split = SHORT[case]
    m = Mix(dev, hq, hkv, q_len, kv_len, window, sinks, kv8, seed=case)
    for dtype in (BF16, FP32):
        for tn in (None, D.dlfp_tuning(split or 0)):
            m.check(m.run(ws, dtype, SCALE, tn), SCALE, rows=[0, 399, 795, 799])
    assert D.dlfp_workspace_error(ws.buf) == 0


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("kv_len", [[700, 5, 1, 20], [300, 700, 31, 290], [20, 700, 3, 17, 9, 1, 2]])
def test_few_decoders_beside_many_prefill_units(dev, ws, kv_len, kv8):
    """More prefill units than lead the grid, and fewer decode workgroups than a group of it."""
    q_len = [600 if n == 700 else 1 for n in kv_len]
    m = Mix(dev, 16, 2, q_len, kv_len, None, 0, kv8, seed=len(kv_len))
    for dtype in (BF16, FP32):
        b = m.batch(D.dlfp_tuning(64, 64, 0, 16))
        assert b.meta.num_prefill_units > 256
        m.check(m.run(ws, dtype, SCALE, batch=b), SCALE, rows=[0, 255, 599])
    assert D.dlfp_workspace_error(ws.buf) == 0
