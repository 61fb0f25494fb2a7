"""Windowed metadata, refusals and oracle pins of dlfp_cache.h (no GPU needed).

The work list is checked against its definition: every (row, key) pair that the
mask lets through is read by exactly one unit, and only pages with such a key.
The oracle's e4m3 codes are pinned by torch's type, its rotation by complex
numbers, its windowed rows by the full mask of oracle.attention.
"""
import ctypes
import os
import re
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from oracle import attention as oa
from oracle import window as ow
from paper_2609_38386_amd import dlfp as D
from paper_2609_38386_amd import runtime as rt

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DIMS = D.make_dims(16, 8)


def test_library_exports_every_declared_symbol():
    txt = open(os.path.join(ROOT, "include", "dlfp_cache.h")).read()
    txt = re.sub(r"/\*.*?\*/", "", txt, flags=re.S)
    declared = set(re.findall(r"\bint\s+(dlfp_\w+)\s*\(", txt))
    assert declared == set(D.CACHE_EXPORTS)
    for name in declared:
        assert hasattr(D.lib(), name), name


def _table(kv_len, window=None, sinks=0, q_len=None, seed=0):
    """Pages in sight only, the others -1."""
    rng = np.random.default_rng(seed)
    width = max(-(-n // 16) for n in kv_len)
    table = np.full((len(kv_len), width), -1, np.int32)
    order = iter(rng.permutation(sum(-(-n // 16) for n in kv_len)))
    for s, n in enumerate(kv_len):
        rows = np.arange(n - q_len[s], n)
        for p in range(-(-n // 16)):
            key = np.arange(16 * p, min(16 * p + 16, n))
            if ow.sees(rows[:, None], key[None], window, sinks).any():
                table[s, p] = next(order)
    return table, sum(-(-n // 16) for n in kv_len)


MIXES = [
    ([1], [1], None, 0), ([1], [1], 1, 0), ([1, 1, 1], [5, 16, 17], 1, 1),
    ([1] * 6, [64, 65, 700, 1000, 1, 4096], 128, 4), ([1] * 4, [5000, 5001, 30, 8000], 4096, 64),
    ([40, 1, 1], [40, 300, 77], 32, 4), ([200, 3, 1], [900, 3, 1200], 17, 33),
    ([130, 129], [130, 1000], None, 0), ([64, 2], [4000, 17], 100, 5), ([33], [2000], 1, 0),
    ([300], [301], 2 ** 31 - 1, 2 ** 31 - 1), ([7, 1], [50, 50], 3, 48), ([], [], 5, 5),
]


@pytest.mark.parametrize("hq,hkv", [(16, 8), (8, 8), (8, 1), (4, 1)])
@pytest.mark.parametrize("case", range(len(MIXES)))
def test_window_list(case, hq, hkv):
    q_len, kv_len, window, sinks = MIXES[case]
    dims = D.make_dims(hq, hkv)
    table, blocks = (_table(kv_len, window, sinks, q_len) if q_len else
                     (np.zeros((0, 1), np.int32), 1))
    w = D.dlfp_window(window, sinks) if window is not None else None
    for tn in [None, D.dlfp_tuning(16, 64), D.dlfp_tuning(128, 512, 0, 5), D.dlfp_tuning(0, 0, 64),
               D.dlfp_tuning(0, 0, 0, 1)]:
        meta = D.dlfp_build_window_meta(dims, q_len, kv_len, table, blocks, w, tn)
        ow.check_window_list(meta, q_len, kv_len, hq, hkv, window, sinks)
        cu = np.concatenate([[0], np.cumsum(q_len)]).astype(int)
        assert meta.cu_q[:len(q_len) + 1].tolist() == cu.tolist()
        slots = [table[s, p // 16] * 16 + p % 16 for s in range(len(q_len))
                 for p in range(kv_len[s] - q_len[s], kv_len[s])]
        assert meta.slot_mapping[:meta.num_tokens].tolist() == slots
        assert meta.num_append == 0 and meta.decode_pages_in_flight == 3


def test_window_meta_refusals():
    table = np.arange(8, dtype=np.int32).reshape(2, 4)

    def status(q=(1, 3), kv=(20, 50), t=table, blocks=8, w=D.dlfp_window(16, 4), dims=DIMS, tn=None):
        try:
            D.dlfp_build_window_meta(dims, list(q), list(kv), t, blocks, w, tn)
            return 0
        except D.DlfpError as e:
            return e.status

    assert status() == 0 and status(w=None) == 0
    assert status(w=D.dlfp_window(0, 4)) == -1 and status(w=D.dlfp_window(4, -1)) == -1
    assert status(q=(0, 3)) == -1 and status(q=(21, 3)) == -1
    assert status(kv=(20, 65)) == -2                     # more pages than the table has
    assert status(blocks=7) == -2                        # a block id past the pool
    assert status(blocks=2 ** 27 + 1) == -2              # slots past 32 bits
    assert status(dims=D.make_dims(16, 8, head_dim=64)) == -5
    assert status(dims=D.make_dims(24, 8)) == -5
    assert status(tn=D.dlfp_tuning(24)) == -1 and status(tn=D.dlfp_tuning(0, 32)) == -1
    # Dropped pages are not looked at; pages in sight and of new tokens are.
    far = np.array([[0, -1, -1, 1]], np.int32)
    assert status((1,), (50,), far, 2, D.dlfp_window(2, 4)) == 0
    assert status((1,), (50,), far, 2, D.dlfp_window(3, 4)) == -2
    assert status((1,), (50,), far, 2, D.dlfp_window(2, 17)) == -2
    assert status((3,), (50,), far, 2, D.dlfp_window(1, 4)) == -2
    assert status((1,), (50,), far, 2, None) == -2


def test_metadata_kinds_are_refused_where_the_other_belongs():
    """Counts and kinds are checked before any pointer, so no device is needed."""
    L = D.lib()
    table = np.arange(4, dtype=np.int32).reshape(1, 4)
    windowed = D.dlfp_build_window_meta(DIMS, [1], [50], table, 4)
    plain = D.dlfp_build_varlen_meta(DIMS, [1], [50], table, 4)
    none, one = None, ctypes.c_void_p(16)
    args = (one, one, 4, 4, one, one, one)
    rest = (0.1, one, 0, one, 1 << 24, none)
    assert L.dlfp_attention_window(DIMS, plain.c, *args, *rest) == -1
    assert L.dlfp_attention_kv8(DIMS, plain.c, *args, one, one, *rest) == -1
    assert L.dlfp_attention_mixed(DIMS, windowed.c, *args, *rest) == -1
    # Null pointers, scale, output type, workspace.
    assert L.dlfp_attention_window(DIMS, windowed.c, none, *args[1:], *rest) == -1
    assert L.dlfp_attention_kv8(DIMS, windowed.c, *args, none, one, *rest) == -1
    for bad, want in [((0.0, one, 0, one, 1 << 24, none), -1), ((0.1, one, 2, one, 1 << 24, none), -1),
                      ((0.1, one, 0, one, 1000, none), -3), ((float("nan"), one, 0, one, 1 << 24, none), -1),
                      ((0.1, none, 0, one, 1 << 24, none), -1),
                      ((0.1, ctypes.c_void_p(24), 0, one, 1 << 24, none), -1),
                      ((0.1, one, 0, ctypes.c_void_p(8), 1 << 24, none), -1)]:
        assert L.dlfp_attention_window(DIMS, windowed.c, *args, *bad) == want
        assert L.dlfp_attention_kv8(DIMS, windowed.c, *args, one, one, *bad) == want
    empty = D.dlfp_build_window_meta(DIMS, [], [], np.zeros((0, 1), np.int32), 1)
    assert L.dlfp_attention_window(DIMS, empty.c, *([none] * 2), 1, 1, none, none, none, 0.1, none,
                                   0, none, 0, none) == 0
    assert L.dlfp_attention_kv8(DIMS, empty.c, *([none] * 2), 1, 1, none, none, none, none, none,
                                0.1, none, 0, none, 0, none) == 0


def test_append_refusals():
    """Every argument is checked before a launch, so no device is needed."""
    L = D.lib()
    one = ctypes.c_void_p(256)

    def status(dims=DIMS, rope=(256, 100, 128, 0), n=3, p=one, s=one, q=one, ldq=2048, k=one,
               ldk=1024, v=one, ldv=1024, o=one, ldo=2048, kc=one, vc=one, ke=one, blocks=4):
        r = D.dlfp_rope(*rope) if rope else None
        a = (dims, r, n, p, s, q, ldq, k, ldk, v, ldv, o, ldo, kc, vc)
        got = {L.dlfp_rope_append_kv8(*a, ke, ke, blocks, None)}
        if ke is one:
            got.add(L.dlfp_rope_append(*a, blocks, None))
        assert len(got) == 1
        return got.pop()

    assert status(n=0) == 0
    assert status(n=0, p=None, s=None, q=None, k=None, v=None, o=None, kc=None, vc=None,
                  rope=(0, 0, 128, 0)) == 0
    for bad in [dict(n=-1), dict(rope=None), dict(rope=(256, 100, 128, 2)), dict(rope=(0, 100, 128, 0)),
                dict(rope=(256, 0, 128, 0)), dict(rope=(260, 100, 128, 0)), dict(p=None), dict(s=None),
                dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(kc=None), dict(vc=None),
                dict(ke=None), dict(blocks=-1), dict(ldq=2047), dict(ldq=2040), dict(ldk=1028),
                dict(ldv=1016), dict(ldo=1024), dict(q=ctypes.c_void_p(264)),
                dict(kc=ctypes.c_void_p(264))]:
        assert status(**bad) == -1, bad
    for bad in [dict(rope=(256, 100, 96, 0)), dict(rope=(256, 100, 0, 0)), dict(rope=(256, 100, 256, 0)),
                dict(dims=D.make_dims(16, 8, page_size=32)), dict(dims=D.make_dims(24, 8))]:
        assert status(**bad) == -5, bad


def test_binding_refusals():
    q = torch.zeros((3, 16, 128), dtype=torch.bfloat16)
    k = torch.zeros((3, 8, 128), dtype=torch.bfloat16)
    at = torch.zeros(3, dtype=torch.int32)
    rope, pool = rt.Rope(10, "cpu"), rt.KVPool8(4, 8, "cpu")
    for bad in [(q.transpose(0, 1), k, k, q), (q, k[:2], k, q), (q.float(), k, k, q),
                (q, k[:, :4], k, q)]:
        with pytest.raises(ValueError):
            rt.rope_append(DIMS, rope, pool, at, at, *bad)
    with pytest.raises(ValueError):
        rt.rope_append(DIMS, rope, pool, at.long(), at, q, k, k, q)
    with pytest.raises(ValueError):   # on the host
        rt.rope_append(DIMS, rope, pool, at, at, q, k, k, q)
    with pytest.raises(ValueError):   # every other position
        rt.rope_append(DIMS, rope, pool, torch.zeros(6, dtype=torch.int32)[::2], at, q, k, k, q)
    batch = rt.WindowBatch(DIMS, [3], [3], np.zeros((1, 1), np.int32), 1, "cpu")
    ws = SimpleNamespace(ensure=lambda *a: torch.zeros(1 << 20, dtype=torch.uint8))
    for bad in [(q, q), (q[:2], q), (q, q.float()[:, :8]), (q.transpose(0, 1), q)]:
        with pytest.raises(ValueError):
            batch.attention(pool, bad[0], 0.1, bad[1], ws)
    with pytest.raises(ValueError):
        rt.KVPool8.of(pool.k, pool.v, pool.k_exp[:2], pool.v_exp)
    with pytest.raises(ValueError):
        rt.KVPool.of(pool.k, pool.v)
    with pytest.raises(ValueError):
        rt.WindowBatch(DIMS, [1], [5], np.zeros((1, 1), np.int32), 1, "cpu", sinks=4)


# ------------------------------------------------------------------ oracle pins

def test_oracle_e4m3_against_torch():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(ow.E4M3, want, equal_nan=True)
    rng = np.random.default_rng(1)
    x = np.concatenate([rng.normal(size=4000) * 2.0 ** rng.integers(-12, 8, 4000),
                        (ow.E4M3[:126] + ow.E4M3[1:127]) / 2, ow.E4M3[:127], [0.0, -0.0]])
    x = np.clip(x, -448, 448).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ow.e4m3_encode(x), want)
    assert ow.e4m3_encode([np.inf, np.nan, -np.inf]).tolist() == [127, 127, 255]
    with pytest.raises(ValueError):
        ow.e4m3_encode([449.0])


def test_oracle_page_exponent_is_the_least():
    for a in [448.0, 449.0, 1e-3, 7.0, 1.75 * 2.0 ** 20, 1.7500001 * 2.0 ** 20, 3e38, 2.0 ** -95]:
        e = ow.page_exponent(a)
        assert a <= 448 * 2.0 ** e and (e == -100 or a > 448 * 2.0 ** (e - 1))
    assert ow.page_exponent(0.0) == -100 and ow.page_exponent(2.0 ** -130) == -100


def test_oracle_append_page_by_hand():
    codes = np.zeros((16, 2), np.uint8)
    codes, e = ow.append_page(codes, 0, [[448.0, -1.0]], 0)
    assert e == 127 and ow.E4M3[codes[0]].tolist() == [448.0, -1.0]
    # A token of twice the range: the older codes halve.
    codes, e = ow.append_page(codes, e, [[896.0, 0.0]], 1)
    assert e == 128 and (ow.E4M3[codes[:2]] * 2).tolist() == [[448.0, -1.0], [896.0, 0.0]]
    # A smaller one leaves them; slot 0 begins anew; NaN and infinities do not count.
    codes, e = ow.append_page(codes, e, [[2.0, np.inf]], 2)
    assert e == 128 and ow.E4M3[codes[2, 0]] == 1.0 and np.isnan(ow.E4M3[codes[2, 1]])
    codes, e = ow.append_page(codes, e, [[3.5, np.nan]], 0)
    assert e == 120 and ow.E4M3[codes[0, 0]] == 448.0
    assert ow.E4M3[codes[1]].tolist() == [448.0, 0.0]    # codes past the new ones stay


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("r", [32, 64, 128])
def test_oracle_rotation_against_complex_numbers(r, interleaved):
    rng = np.random.default_rng(r)
    x = rng.normal(size=(3, 2, 128))
    rope = rt.Rope(20, "cpu", theta=1e4, rotary_dim=r, interleaved=interleaved)
    pos = [0, 19, 7]
    got = ow.rotate(x, rope.table.double().numpy(), pos, interleaved)
    for t, p in enumerate(pos):
        angle = p * 1e4 ** (-2.0 * np.arange(r // 2) / r)
        a, b = (x[t, :, 0:r:2], x[t, :, 1:r:2]) if interleaved else \
            (x[t, :, :r // 2], x[t, :, r // 2:r])
        z = (a + 1j * b) * np.exp(1j * angle)
        ga, gb = (got[t, :, 0:r:2], got[t, :, 1:r:2]) if interleaved else \
            (got[t, :, :r // 2], got[t, :, r // 2:r])
        # the table is rounded to fp32: 2^-24 of each factor
        assert np.abs(ga - z.real).max() <= 1e-6 and np.abs(gb - z.imag).max() <= 1e-6
        assert np.array_equal(got[t, :, r:], x[t, :, r:])


def test_oracle_window_against_the_full_mask():
    rng = np.random.default_rng(5)
    q, k, v = rng.normal(size=(6, 4, 8)), rng.normal(size=(30, 2, 8)), rng.normal(size=(30, 2, 8))
    pos = [24, 25, 26, 27, 28, 29]
    want = oa.attention_rows(q, k, v, 0.3, pos)
    assert np.abs(ow.attention_rows(q, k, v, 0.3, pos) - want).max() < 1e-12
    assert np.abs(ow.attention_rows(q, k, v, 0.3, pos, 30) - want).max() < 1e-12
    assert np.abs(ow.attention_rows(q, k, v, 0.3, pos, 1, 30) - want).max() < 1e-12
    # A window of n keys is the full mask over a sequence cut to them.
    for i, p in enumerate(pos):
        cutk, cutv = (np.concatenate([x[:3], x[p - 4:p + 1]]) for x in (k, v))
        want = oa.attention_rows(q[i:i + 1], cutk, cutv, 0.3, [7])
        kk, vv = k.copy(), v.copy()
        kk[3:p - 4], vv[3:p - 4] = np.nan, np.inf         # what the row does not see
        got = ow.attention_rows(q[i:i + 1], kk, vv, 0.3, [p], 5, 3)
        assert np.abs(got - want).max() < 1e-12
