"""Batches over paged caches of both kinds, for the tests of windowed and 8-bit attention.

A Mix holds the logical queries, keys and values of its sequences (float64, what
the oracle reads) and the caches that hold them: pages in a random order, pages
out of sight left out of the block table, every slot that no row of its sequence
sees poisoned with NaN.
"""
import numpy as np
import torch

from oracle import window as ow
from paper_2609_38386_amd import dlfp as D
from paper_2609_38386_amd import runtime as rt

NAN_CODE = 0x7F


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(torch.bfloat16)


class Mix:
    def __init__(self, dev, hq, hkv, q_len, kv_len, window, sinks, kv8, seed=0, spread=1.0,
                 spare=3, first_block=0, v_exps=None):
        rng = np.random.default_rng(seed)
        self.hq, self.hkv, self.window, self.sinks, self.kv8 = hq, hkv, window, sinks, kv8
        self.q_len, self.kv_len = list(q_len), list(kv_len)
        self.dims = D.make_dims(hq, hkv)
        pages = [-(-n // 16) for n in kv_len]
        blocks = sum(pages) + spare
        order = iter(rng.permutation(blocks))
        self.table = np.full((len(kv_len), max(pages)), -1, np.int32)
        self.q, self.k, self.v = [], [], []
        shape = (blocks, hkv, 16, 128)
        if kv8:
            pool = [np.full(shape, NAN_CODE, np.uint8) for _ in "kv"]
            exps = [np.full(shape[:2], 127, np.uint8) for _ in "kv"]
        else:
            pool = [np.full(shape, np.nan, np.float32) for _ in "kv"]
        for s, (ql, kl) in enumerate(zip(q_len, kv_len)):
            self.q.append(bf16(rng.normal(size=(ql, hq, 128)) * spread).double().numpy())
            rows = np.arange(kl - ql, kl)
            seen = ow.sees(rows[:, None], np.arange(kl)[None], window, sinks).any(0)
            at = np.flatnonzero(np.add.reduceat(seen, np.arange(0, kl, 16)))
            self.table[s, at] = [next(order) for _ in at]
            for x, (name, cache) in enumerate(zip("kv", pool)):
                data = rng.normal(size=(kl, hkv, 128))
                if kv8:
                    e = rng.integers(-9, -4, size=(pages[s], hkv))
                    if name == "v" and v_exps:   # pages of far scales, all of them full
                        e = rng.choice(v_exps, size=(pages[s], hkv))
                        data *= np.repeat(2.0 ** (e + 7), 16, 0)[:kl, :, None]
                    scale = np.repeat(2.0 ** e, 16, 0)[:kl, :, None]
                    codes = ow.e4m3_encode(np.clip(data / scale, -448, 448))
                    data = ow.E4M3[codes] * scale
                    codes[~seen] = NAN_CODE
                    for p in at:
                        exps[x][self.table[s, p]] = e[p] + 127
                else:
                    codes = bf16(data).float().numpy()
                    data = codes.astype(np.float64)
                    codes[~seen] = np.nan
                getattr(self, name).append(data)
                for p in at:
                    page = codes[16 * p:16 * p + 16]
                    cache[self.table[s, p], :, :len(page)] = page.transpose(1, 0, 2)
        swap = [(t & 3) | ((t & 4) << 1) | ((t & 8) >> 1) for t in range(16)]
        pool[1] = np.ascontiguousarray(pool[1][:, :, swap].transpose(0, 1, 3, 2))
        if kv8:
            k, v = (torch.from_numpy(x).to(dev).view(torch.float8_e4m3fn) for x in pool)
            ke, ve = (torch.from_numpy(x).to(dev) for x in exps)
        else:
            k, v = (bf16(x).to(dev) for x in pool)
        if first_block:  # the same pages far into a larger pool
            def far(x):
                big = torch.empty((first_block + blocks, *x.shape[1:]), dtype=torch.uint8 if kv8
                                  else x.dtype, device=dev)
                big[first_block:] = x.view(big.dtype)
                return big.view(x.dtype)
            k, v = far(k), far(v)
            if kv8:
                ke, ve = far(ke), far(ve)
            self.table[self.table >= 0] += first_block
        self.blocks = first_block + blocks
        self.v_exp = max(v_exps) if v_exps else -5   # the largest exponent drawn
        self.pool = rt.KVPool8.of(k, v, ke, ve) if kv8 else rt.KVPool.of(k, v)
        self.dq = bf16(np.concatenate(self.q)).to(dev)
        self.dev = dev

    def batch(self, tuning=None):
        return rt.WindowBatch(self.dims, self.q_len, self.kv_len, self.table, self.blocks, self.dev,
                              self.window, self.sinks, tuning)

    def run(self, workspace, dtype, scale, tuning=None, batch=None):
        out = torch.full(self.dq.shape, float("nan"), dtype=dtype, device=self.dev)
        (batch or self.batch(tuning)).attention(self.pool, self.dq, scale, out, workspace)
        return out

    def check(self, out, scale, rows=None):
        """Every element within its bound of the oracle's.

        With p_j the weights of a row and A = sum_j p_j |v_j - o| an element's spread,
        a relative error d of every weight moves the element by at most 2 d A / (1 - d)
        (numerator and denominator).  d: the score's error, 128 products summed in fp32,
        at most 128 steps of 2^-24 of sum |q k| scale; 2^-18 for the exponential (its
        argument, up to 2^5, rounded to 2^-24 of it, and its own last place) and the
        sums over keys; the weights' rounding: one bf16 term 2^-8 (prompts, bf16
        output), two 2^-15, three 2^-21.  Then the output's half step.

        What does not fall with the spread, where one key has all the weight: roundings of
        the sum itself, each at most 2^-24 of B = sum_j p_j |v_j|.  A matrix product adds
        16 keys or more, so n keys take n / 16; the three terms of a weight leave 2^-22 of
        it (two cut to 8 bits, the third rounded to 8: 2^-7 2^-7 2^-8), four such; the
        exponentials of the wavefronts' and splits' maxima, their sums, the division and
        the product with it, up to 12 more.

        Weights are 32-bit numbers: an exponential below 2^-126 is 0, of the weight itself or
        of a wavefront's or split's maximum against the others'.  A reference is at most 2^8
        below its maximum, so weights up to 2^-118 of the row's largest may be lost, and of
        three terms each another 2^-126: n 2^-117 of the largest weight times the largest
        value in all.

        8-bit pages with bf16 output: a product of codes adds its 64 or 128 terms to
        within 2^-15 of sum |q k| (2^-15.9 measured over random rows).  A decoder's
        weights (times 2^e of the page's values, relative to the largest) are two e4m3
        terms: 2^-8 of the weight, or, below 2^-6 of the largest such, half of the lesser
        term's least step, 2^-15 of the largest, each times a value of at most 448 2^e."""
        got = out.double().cpu().numpy()
        assert np.isfinite(got).all()
        half = 2.0 ** -8 if out.dtype == torch.bfloat16 else 2.0 ** -24
        at = 0
        for s, (ql, kl) in enumerate(zip(self.q_len, self.kv_len)):
            pick = np.arange(ql) if rows is None else np.unique(np.clip(rows, 0, ql - 1))
            pos = kl - ql + pick
            for h in range(self.hkv):
                hs = slice(h * self.hq // self.hkv, (h + 1) * self.hq // self.hkv)
                seen = ow.sees(pos[:, None], np.arange(kl)[None], self.window, self.sinks)
                keep = seen.any(0)
                k, v, seen = self.k[s][keep, h], self.v[s][keep, h], seen[:, keep]
                for i, r in enumerate(pick):
                    q = self.q[s][r, hs]
                    kk, vv = k[seen[i]], v[seen[i]]
                    sc = scale * (q @ kk.T)
                    w = np.exp(sc - sc.max(1, keepdims=True))
                    w /= w.sum(1, keepdims=True)
                    o = w @ vv
                    spread = np.stack([(w[j][:, None] * np.abs(vv - o[j])).sum(0)
                                       for j in range(len(q))])
                    d = 128 * 2.0 ** -24 * scale * (np.abs(q) @ np.abs(kk).T).max() + 2.0 ** -18
                    least = 0.0
                    if half < 2.0 ** -20:
                        d += 2.0 ** -21
                    else:
                        d += 2.0 ** -8 if ql > 1 or self.kv8 else 2.0 ** -15
                        if self.kv8:
                            d += 2.0 ** -15 * scale * (np.abs(q) @ np.abs(kk).T).max()
                            if ql == 1:
                                least = 2.0 ** -15 * len(vv) * w.max(1, keepdims=True) * \
                                    448 * 2.0 ** self.v_exp
                    sums = (len(vv) / 16 + 16) * 2.0 ** -24 * (w @ np.abs(vv))
                    lost = len(vv) * 2.0 ** -117 * w.max(1, keepdims=True) * np.abs(vv).max()
                    tol = least + half * np.abs(o) + 2 * d / (1 - d) * spread + sums + lost + 1e-30
                    err = np.abs(got[at + r, hs] - o)
                    assert (err <= tol).all(), (s, r, h, float((err / tol).max()))
            at += ql
