"""The bounds of _rows reject outputs that are wrong (no GPU needed)."""
import math

import numpy as np
import pytest

from _rows import far_scales, one_dominates

SCALE = 1.0 / math.sqrt(128)


def _bf16(x):
    return x * (1 + 2.0 ** -9)   # any value within half a step


@pytest.mark.parametrize("weight", [0.5, 0.9, 0.99, 0.9999])
@pytest.mark.parametrize("n", [512, 4096])
def test_lost_weights_are_rejected(n, weight):
    m = one_dominates(1, 3, 4, 2, n, weight, 1.0, "cpu", device_pool=False)
    want, (bf16, fp32) = m.expected(SCALE)
    first = np.exp(SCALE * (m.q[:, :2] @ m.k[0, 0]))        # of two heads' first key
    rest = np.exp(SCALE * (m.q[:, :2] @ m.k[1:, 0].T)).sum(-1)
    assert np.all(np.abs(first / (first + rest) - weight) < 0.3 * weight * (1 - weight) + 1e-4)
    assert (np.abs(_bf16(want) - want) <= bf16).all()
    for wrong in (0.9 * want, 0.99 * want, 0.0 * want):
        assert (np.abs(wrong - want) > bf16).mean() > 0.99
    assert (np.abs(_bf16(want) - want) > fp32).mean() > 0.9


def test_wrong_small_scales_are_rejected():
    m = far_scales(2, 24, 8, 4, 900, "cpu", 600.0, device_pool=False)
    want, (bf16, _) = m.expected(SCALE)
    size = np.abs(want).max(2)                               # of each row and head
    assert (size < 1e-6).sum() >= 5 and (size > 1e6).sum() >= 5
    assert (np.abs(_bf16(want) - want) <= bf16).all()
    small = np.where((size < 1e-3)[..., None], 0.0, want)
    wrong = (np.abs(small - want) > bf16).any(2)
    # (Where two keys of far scales have nearly one score, that score's error is allowed
    # to decide.)
    assert not wrong[size >= 1e-3].any() and wrong[size < 1e-3].mean() > 0.85
    assert (np.abs(0.9 * want - want) > bf16).any(2).mean() > 0.9
