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
