"""Decode rows over 8-bit pages from logical codes, and what a row's output may be off by.

Eight_bit holds sequences of one new token each that share their pages: codes and
exponents as given, the float64 values that they stand for beside them.
"""
import numpy as np
import torch

from _paged_mixes import bf16
from oracle import window as ow
from paper_2609_38386_amd import dlfp as D
from paper_2609_38386_amd import runtime as rt

SWAP = [(t & 3) | ((t & 4) << 1) | ((t & 8) >> 1) for t in range(16)]


class EightBit:
    def __init__(self, dev, q, k, v, k_exp, v_exp, seed=0, device_pool=True):
        """q [sequences][hq][128]; k, v codes [n][hkv][128]; k_exp, v_exp bytes [pages][hkv]."""
        self.q = bf16(q).double().numpy()
        n, hkv, _ = k.shape
        pages = -(-n // 16)
        scale = [np.repeat(2.0 ** (e.astype(np.float64) - 127), 16, 0)[:n, :, None]
                 for e in (k_exp, v_exp)]
        self.k, self.v = ow.E4M3[k] * scale[0], ow.E4M3[v] * scale[1]
        self.hq, self.hkv, self.n, self.dev = q.shape[1], hkv, n, dev
        order = np.random.default_rng(seed).permutation(pages + 2)[:pages].astype(np.int32)
        self.table = np.tile(order, (len(q), 1))
        self.blocks = pages + 2
        if not device_pool:
            return
        pool = []
        for codes, rows in ((k, True), (v, False)):
            x = np.full((self.blocks, hkv, 16, 128), 0x7F, np.uint8)
            for p in range(pages):
                page = codes[16 * p:16 * p + 16].transpose(1, 0, 2)
                x[order[p], :, :page.shape[1]] = page
            x = x if rows else np.ascontiguousarray(x[:, :, SWAP].transpose(0, 1, 3, 2))
            pool.append(torch.from_numpy(x).to(dev).view(torch.float8_e4m3fn))
        for e in (k_exp, v_exp):
            x = np.full((self.blocks, hkv), 127, np.uint8)
            x[order] = e
            pool.append(torch.from_numpy(x).to(dev))
        self.pool = rt.KVPool8.of(*pool)
        self.dq = bf16(q).to(dev)

    def run(self, workspace, dtype, scale, tuning=None, before=None):
        """(output of the decode rows, decode units, prefill units); `before`: (queries of a
        prompt over the same pages, its first position + its length)."""
        q, q_len, kv_len, table = self.dq, [1] * len(self.q), [self.n] * len(self.q), self.table
        if before is not None:
            rows = before.shape[0]
            q = torch.cat([before, q])
            q_len, kv_len = [rows] + q_len, [self.n] + kv_len
            table = np.concatenate([table[:1], table])
        batch = rt.WindowBatch(D.make_dims(self.hq, self.hkv), q_len, kv_len, table, self.blocks,
                               self.dev, tuning=tuning)
        out = torch.full(q.shape, float("nan"), dtype=dtype, device=self.dev)
        batch.attention(self.pool, q, scale, out, workspace)
        m = batch.meta
        return out[len(out) - len(self.q):], m.num_units - m.num_prefill_units, m.num_prefill_units

    def expected(self, scale):
        """(outputs [sequences][hq][128], bounds for bf16 and for fp32 output).

        As _paged_mixes.Mix.check: a relative error d of every weight moves an element by at
        most 2 d / (1 - d) of its spread.  d: 128 products summed in fp32, and, with bf16
        output, the matrix cores' sum to within 2^-15 of sum |q k| (2^-15.9 measured) and
        what the two codes of a query leave, 2^-22 of its row's largest times sum |k|; the
        exponential and the sums 2^-18; the weights' terms: two of bf16 (8 bits cut off,
        the rest rounded to 8) 2^-7 2^-8 with bf16 output, three 2^-21.  No term is relative
        to the row's largest weight, so that many small weights keep theirs together.  Then
        roundings of the sums themselves, weights below 2^-118 of the largest, which may be
        lost, and the output's half step."""
        g = self.hq // self.hkv
        want, bounds = np.empty(self.q.shape), [np.empty(self.q.shape) for _ in range(2)]
        for h in range(self.hq):
            k, v, q = self.k[:, h // g], self.v[:, h // g], self.q[:, h]
            sc = scale * (q @ k.T)
            w = np.exp(sc - sc.max(1, keepdims=True))
            w /= w.sum(1, keepdims=True)
            want[:, h] = o = w @ v
            spread = np.stack([w[i] @ np.abs(v - o[i]) for i in range(len(q))])
            most = scale * (np.abs(q) @ np.abs(k).T).max(1, keepdims=True)
            lost = scale * 2.0 ** -22 * np.abs(q).max(1, keepdims=True) * np.abs(k).sum(1).max()
            sums = (self.n / 16 + 16) * 2.0 ** -24 * (w @ np.abs(v))
            sums += self.n * 2.0 ** -117 * w.max(1, keepdims=True) * np.abs(v).max()
            d = 128 * 2.0 ** -24 * most + 2.0 ** -18
            for i, (half, more) in enumerate(((2.0 ** -8, 2.0 ** -15 * most + lost + 2.0 ** -15),
                                              (2.0 ** -24, 2.0 ** -21))):
                e = d + more
                bounds[i][:, h] = half * np.abs(o) + 2 * e / (1 - e) * spread + sums + 1e-30
        return want, bounds


def one_dominates(seed, rows, hq, hkv, n, weight, spread, dev, **more):
    """Rows whose first key has about `weight` of them and a value of zero; the others'
    scores differ by about `spread`, their values are about 1."""
    rng = np.random.default_rng(seed)
    pages = -(-n // 16)
    u = rng.choice([-1.0, 1.0], size=128)
    logit = np.log(weight / (1 - weight) * (n - 1))
    q = u + rng.normal(size=(rows, hq, 128)) * 0.05
    k = rng.normal(size=(n, hkv, 128)) * spread
    k -= (k @ u)[..., None] * u / 128                # nothing along u
    k[0] = u * logit / np.sqrt(128.0)
    v = 1.0 + 0.3 * rng.normal(size=(n, hkv, 128))
    v[0] = 0.0
    exps = rng.integers(120, 122, size=(2, pages, hkv)).astype(np.uint8)
    codes = [ow.e4m3_encode(np.clip(x / np.repeat(2.0 ** (e.astype(np.float64) - 127), 16, 0)[:n, :, None],
                                    -448, 448)) for x, e in zip((k, v), exps)]
    return EightBit(dev, q, *codes, *exps, seed, **more)


def far_scales(seed, rows, hq, hkv, n, dev, sharp=40.0, **more):
    """Rows whose weight lies on one page or few, value pages in scales up to 2^80 apart."""
    rng = np.random.default_rng(seed)
    pages = -(-n // 16)
    q = rng.normal(size=(rows, hq, 128)) * sharp
    k = rng.normal(size=(n, hkv, 128))
    k_exp = np.full((pages, hkv), 121, np.uint8)
    v_exp = (127 + rng.choice([-40, -15, 0, 40], size=(pages, hkv))).astype(np.uint8)
    codes = [ow.e4m3_encode(np.clip(k * 64.0, -448, 448)),
             ow.e4m3_encode(np.clip(rng.normal(size=(n, hkv, 128)) * 100.0, -448, 448))]
    return EightBit(dev, q, *codes, k_exp, v_exp, seed, **more)
