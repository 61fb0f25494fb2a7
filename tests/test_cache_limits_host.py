"""Sizes at the limits of the rotating appends (no GPU needed: refused before any pointer)."""
import ctypes

import pytest

from paper_2609_38386_amd import dlfp as D


def _status(n, hq, hkv):
    L, one = D.lib(), ctypes.c_void_p(256)
    rope = D.dlfp_rope(256, 100, 128, 0)
    # The null queries are looked at after the counts.
    a = (D.make_dims(hq, hkv), rope, n, one, one, None, 128 * hq, one, 128 * hkv, one, 128 * hkv,
         one, 128 * hq, one, one)
    got = {L.dlfp_rope_append(*a, 4, None), L.dlfp_rope_append_kv8(*a, one, one, 4, None)}
    assert len(got) == 1
    return got.pop()


@pytest.mark.parametrize("hq,hkv", [(1, 1), (8, 1), (16, 8), (64, 8), (17, 17)])
def test_a_launch_stays_below_two_to_the_32_threads(hq, hkv):
    """16 threads for a token and KV head, 64 for a token and group of 16 query heads."""
    each = 16 * hkv + 64 * -(-hq // 16)
    most = 2 ** 32 // each
    assert _status(most - 64, hq, hkv) == -1       # counted as possible: the null pointer is next
    assert _status(most + 64, hq, hkv) == -2
    assert _status(2 ** 31 - 1, hq, hkv) == -2
    # Few tokens of very many heads: 64 threads for each of both.
    heads = 2 ** 32 // (64 * 512)
    assert _status(512, heads // 2, heads // 2) == -1 and _status(512, heads, heads) == -2
