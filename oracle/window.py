"""Attention with a sliding window and sinks, 8-bit pages and the rotation, in float64.

Definitions followed, one by one and without blocking:

* a row at position p sees key j <= p with p - j < window or j < sinks;
* e4m3 codes (OCP): sign, 4 exponent bits of bias 7, 3 mantissa bits; 0x7F and
  0xFF are NaN, there is no infinity; a page's exponent byte e scales its codes
  by 2^(e - 127);
* an append to an 8-bit page: the least E >= -100 with amax <= 448 * 2^E over
  the new tokens' finite magnitudes (at least the page's exponent when older
  tokens stay), codes nearest to x 2^-E with ties to even;
* the rotation: (a, b) -> (a c - b s, b c + a s) for the pairs of the first
  rotary_dim dims.
"""
from __future__ import annotations

import math

import numpy as np

PAGE = 16
EXP_MIN, EXP_BIAS = -100, 127


def sees(pos, key, window, sinks):
    """Whether the row at `pos` sees `key` (scalars or arrays); window None: no window."""
    pos, key = np.asarray(pos), np.asarray(key)
    if window is None:
        return key <= pos
    return (key <= pos) & ((pos - key < window) | (key < sinks))


def attention_rows(q, k, v, scale, positions, window=None, sinks=0):
    """q [R][Hq][D], k, v [n][Hkv][D] float64; keys and values that no row sees may hold
    anything.  Returns [R][Hq][D]."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    n, hkv, _ = k.shape
    g = q.shape[1] // hkv
    pos = np.asarray(positions, np.int64)
    seen = sees(pos[:, None], np.arange(n)[None], window, sinks)
    out = np.empty(q.shape)
    for h in range(q.shape[1]):
        kh, vh = k[:, h // g], v[:, h // g]
        for i in range(len(pos)):
            at = np.flatnonzero(seen[i])
            s = scale * (kh[at] @ q[i, h])
            w = np.exp(s - s.max())
            out[i, h] = (w @ vh[at]) / w.sum()
    return out


# ------------------------------------------------------------------ 8-bit pages

def e4m3_values() -> np.ndarray:
    """The value of each of the 256 codes."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = math.nan if e == 15 and m == 7 else \
            m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[c] = -x if c & 128 else x
    return out


E4M3 = e4m3_values()


def e4m3_encode(x) -> np.ndarray:
    """Codes (uint8) nearest to x, ties to the code with an even mantissa; NaN and
    infinities become NaN.  |x| of finite values is at most 448."""
    x = np.asarray(x, np.float64)
    pos = E4M3[:127]                                   # 0 .. 448, ascending
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    if a.size and a.max() > 448.0:
        raise ValueError("beyond the format")
    hi = np.clip(np.searchsorted(pos, a), 1, 126)      # pos[hi - 1] <= a <= pos[hi]
    lo = hi - 1
    down, up = a - pos[lo], pos[hi] - a
    code = np.where(down < up, lo, np.where(up < down, hi, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(np.isfinite(x), code, 127).astype(np.uint8)
    return code | np.where(np.signbit(x), 128, 0).astype(np.uint8)


def page_exponent(amax: float) -> int:
    if amax == 0.0:
        return EXP_MIN
    m, e = math.frexp(amax)                            # 448 = 0.875 * 2^9
    return max(EXP_MIN, e - 9 if m <= 0.875 else e - 8)


def append_page(codes, exp_byte, x, slot0):
    """One page's token rows ([16][D] uint8 codes of one KV head) with tokens x ([n][D]
    float64) written from slot0 on: (codes, exponent byte)."""
    codes, x = np.array(codes, np.uint8), np.asarray(x, np.float64)
    finite = np.abs(x[np.isfinite(x)])
    e = page_exponent(float(finite.max()) if finite.size else 0.0)
    was = int(exp_byte) - EXP_BIAS
    if slot0 > 0:
        e = max(e, was)
        if e > was:
            codes[:slot0] = e4m3_encode(E4M3[codes[:slot0]] * 2.0 ** (was - e))
    codes[slot0:slot0 + len(x)] = e4m3_encode(x * 2.0 ** -e)
    return codes, e + EXP_BIAS


def rotate(x, table, positions, interleaved=False):
    """x [T][H][D] turned to positions [T]; table [positions][r]: cosines, then sines.
    In the type of x."""
    x, table = np.array(x), np.asarray(table, np.asarray(x).dtype)
    r = table.shape[1]
    for t, p in enumerate(positions):
        for i in range(r // 2):
            i0, i1 = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
            c, s = table[p, i], table[p, r // 2 + i]
            a, b = x[t, :, i0].copy(), x[t, :, i1].copy()
            x[t, :, i0] = a * c - b * s
            x[t, :, i1] = b * c + a * s
    return x


# ------------------------------------------------------------------ the work list

def unit_pages(rec):
    """Pages of the sequence that a unit reads, in its order."""
    vb, ve, sinks, gap = (int(rec[i]) for i in (4, 5, 14, 15))
    sunk = -(-sinks // PAGE) if gap else 0
    return [p + gap if p >= sunk else p for p in range(vb // PAGE, -(-ve // PAGE))]


def check_window_list(meta, q_len, kv_len, num_q_heads, num_kv_heads, window, sinks):
    """Every (row, key) pair that the mask lets through is read by exactly one unit of its
    KV head, no unit reads a page without such a key, and the records' format holds."""
    g = num_q_heads // num_kv_heads
    cu = np.concatenate([[0], np.cumsum(q_len)]).astype(int)
    read, groups, end = {}, {}, (256 + 4 * 65536) // 4
    for i, r in enumerate(meta.work):
        r = [int(x) for x in r]
        s, kh, t0, nt, vb, ve, grp, split, nsplits = r[:9]
        pre = i < meta.num_prefill_units
        assert (q_len[s] > 1) == pre and r[11] == (0 if pre else 1)
        assert nt * g <= 128 and 0 <= t0 and t0 + nt <= q_len[s] and nt >= 1
        assert r[12] == cu[s] + t0 and r[13] == kv_len[s] - q_len[s] + t0
        assert vb % (64 if pre else 16) == 0 and vb < ve
        assert ve - vb <= (32768 if pre and nt * g > 32 else 4096)
        assert r[9] == (window if window is not None else 2 ** 31 - 1)
        assert r[14] == min(sinks, 2 ** 31 - 17) and r[15] >= 0
        first, last = r[13], r[13] + nt - 1
        keys = []
        for p in unit_pages(r):
            assert 0 <= p <= (kv_len[s] - 1) // PAGE
            key = np.arange(p * PAGE, min((p + 1) * PAGE, kv_len[s]))
            rows = np.arange(first, last + 1)
            assert sees(rows[:, None], key[None], window, sinks).any(), (r, p)
            keys.append(key)
        # keys of the last page past the unit's end belong to no unit's range
        virtual = np.arange(vb, ve)
        sunk = -(-r[14] // PAGE) * PAGE if r[15] else 0
        key = np.where(virtual >= sunk, virtual + r[15] * PAGE, virtual)
        assert key[-1] <= last
        for t in range(nt):
            seen = key[sees(first + t, key, window, sinks)]
            read.setdefault((s, t0 + t, kh), []).append(seen)
        if nsplits > 1:
            groups.setdefault(grp, []).append((split, nsplits, r[10], nt * g))
        else:
            assert grp == -1
    for s, (ql, kl) in enumerate(zip(q_len, kv_len)):
        for t in range(ql):
            pos = kl - ql + t
            want = np.flatnonzero(sees(pos, np.arange(kl), window, sinks))
            for kh in range(num_kv_heads):
                got = np.sort(np.concatenate(read.pop((s, t, kh))))
                assert np.array_equal(got, want), (s, t, kh)
    assert not read
    assert sorted(groups) == list(range(meta.num_groups))
    spans = []
    for members in groups.values():
        n, at, rows = members[0][1:]
        assert sorted(m[0] for m in members) == list(range(n))
        assert all(m[1:] == (n, at, rows) for m in members)
        spans.append((at, at + n * (-(-rows * 130 // 64) * 64)))
    for a, b in sorted(spans):
        assert a >= end
        end = b
    assert 4 * end <= meta.workspace_bytes
