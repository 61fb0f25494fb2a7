"""GPU: calls of windowed and 8-bit attention at the ends of what they take."""
import math

import numpy as np
import pytest
import torch

from _paged_mixes import Mix, bf16
from _rows import far_scales, one_dominates
from oracle import window as ow
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


# rows, hq, hkv, keys, decode split, rows of a prompt beside: units of eight wavefronts,
# of four, of one, and of one beside a prompt.
DOMINATED = [(2, 8, 1, 4096, 4096, 0), (40, 8, 2, 4096, 2048, 0), (530, 4, 1, 512, 512, 0),
             (300, 4, 2, 2048, 2048, 1500), (3, 2, 1, 1024, 1024, 0), (520, 1, 1, 300, 304, 0)]


@pytest.mark.parametrize("spread", [0.0, 1.0])
@pytest.mark.parametrize("weight", [0.5, 0.9, 0.99, 0.9999])
@pytest.mark.parametrize("case", range(len(DOMINATED)))
def test_one_key_has_most_of_the_weight(dev, ws, case, weight, spread):
    """The others' weights, each far below the largest, together make the output, whatever
    the number of wavefronts."""
    rows, hq, hkv, n, split, prompt = DOMINATED[case]
    m = one_dominates(case, rows, hq, hkv, n, weight, spread, dev)
    want, bounds = m.expected(SCALE)
    before = m.dq[:1].expand(prompt, -1, -1).contiguous() if prompt else None
    for dtype, tol in zip((BF16, FP32), bounds):
        got, units, prefill = m.run(ws, dtype, SCALE, D.dlfp_tuning(split), before)
        assert (units > 512) == (rows >= 300) and (prefill > 0) == (prompt > 0)
        err = np.abs(got.double().cpu().numpy() - want)
        print(dtype, float(np.linalg.norm(err) / np.linalg.norm(want)), float((err / tol).max()))
        assert (err <= tol).all()
    assert D.dlfp_workspace_error(ws.buf) == 0


@pytest.mark.parametrize("sharp", [40.0, 600.0])
@pytest.mark.parametrize("rows,hq,hkv,n,split", [(6, 8, 4, 900, 0), (3, 8, 1, 4000, 4096),
                                                 (530, 2, 1, 400, 400), (40, 16, 2, 700, 0)])
def test_each_row_by_its_own_scales(dev, ws, rows, hq, hkv, n, split, sharp):
    """Rows whose weight is on value pages of small scales, beside others' of large ones."""
    m = far_scales(rows, rows, hq, hkv, n, dev, sharp)
    want, bounds = m.expected(SCALE)
    for dtype, tol in zip((BF16, FP32), bounds):
        got, _, _ = m.run(ws, dtype, SCALE, D.dlfp_tuning(split))
        assert (np.abs(got.double().cpu().numpy() - want) <= tol).all()


# hq, hkv, q_len, kv_len, window, sinks, tuning: decode units of eight, four and one
# wavefronts, whole and split, alone and beside a prompt; prompts' tiles of 128 and of 32
# rows, whole and in parts of which the last batch of a merge has one to three.
INFINITE = [
    (8, 2, [1, 1], [1500, 900], None, 0, None), (2, 2, [1, 1], [700, 40], None, 0, (64,)),
    (16, 2, [1] * 40, [30 + 25 * i for i in range(40)], None, 0, (2048,)),
    (8, 1, [1] * 530, [1 + i % 90 for i in range(530)], None, 0, None),
    (4, 2, [40, 1, 1], [300, 500, 33], None, 0, None), (4, 1, [1, 1], [800, 90], 200, 20, None),
    (8, 2, [1] * 300 + [1500], [100] * 300 + [1500], None, 0, None),
    (8, 2, [100], [700], None, 0, (0, 0, 0, 32)), (8, 2, [100], [700], None, 0, (0, 128, 0, 32)),
    (2, 2, [100], [900], None, 0, (0, 192, 0, 40)), (2, 2, [60], [900], 800, 16, (0, 64, 0, 60)),
    (8, 2, [9], [900], None, 0, (0, 0, 0, 8)), (16, 2, [9], [900], None, 0, (0, 192, 0, 4)),
    (4, 2, [70], [500], 400, 0, (0, 64, 0, 2)), (8, 2, [33, 2], [300, 80], None, 0, (0, 64)),
]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("case", range(len(INFINITE)))
def test_infinite_values(dev, ws, case, dtype):
    """An infinite value that all rows of a sequence see makes that dim of its heads that
    infinity and leaves every other output as it was."""
    hq, hkv, q_len, kv_len, window, sinks, tn = INFINITE[case]
    m = Mix(dev, hq, hkv, q_len, kv_len, window, sinks, False, seed=case)
    batch, g = m.batch(D.dlfp_tuning(*tn) if tn else None), hq // hkv
    want = m.run(ws, dtype, SCALE, batch=batch)
    assert want.isfinite().all()
    at = 0
    for s, (ql, kl) in enumerate(zip(q_len, kv_len)):
        head, dim, sign = s % hkv, (11 * s + 3) % 128, 1.0 - 2.0 * (s % 2)
        seen = min(kl - ql + 1, window or kl)            # by every row, up to the first one's
        key = kl - ql - (7 * s) % max(1, seen - ql)
        page = m.pool.v[int(m.table[s, key // 16]), head, dim]
        page[SWAP[key % 16]] = sign * math.inf
        want[at:at + ql, head * g:(head + 1) * g, dim] = sign * math.inf
        at += ql
    got = m.run(ws, dtype, SCALE, batch=batch)
    wrong = (got != want).nonzero()[:4].tolist()
    assert not wrong
    assert D.dlfp_workspace_error(ws.buf) == 0


def test_append_of_far_8_bit_pages(dev):
    """Codes and exponents of keys and values in pages past 32 bits of bytes, a run that
    begins inside a page and one that begins the next."""
    hkv, blocks = 8, (1 << 32) // (8 * 2048) + 50
    rng = np.random.default_rng(8)
    sizes = (blocks, hkv, 16, 128), (blocks, hkv, 128, 16), (blocks, hkv), (blocks, hkv)
    pool = rt.KVPool8.of(*(torch.empty(x, dtype=torch.uint8, device=dev) for x in sizes))
    pages = [blocks - 3, blocks - 1]
    codes = rng.integers(0, 120, size=(2, 2, hkv, 16, 128)).astype(np.uint8)
    exps = rng.integers(112, 118, size=(2, 2, hkv)).astype(np.uint8)   # the new tokens' are larger
    for i, b in enumerate(pages):
        pool.k[b] = torch.from_numpy(codes[0, i]).to(dev)
        pool.v[b] = torch.from_numpy(codes[1, i][:, SWAP].swapaxes(1, 2).copy()).to(dev)
        pool.k_exp[b], pool.v_exp[b] = (torch.from_numpy(exps[x, i]).to(dev) for x in range(2))
    n, first = 9, 11                                  # slots 11 .. 15, then 0 .. 3
    qkv = bf16(rng.normal(size=(n, 16 + 2 * hkv, 128)))
    rope = rt.Rope(40, dev)
    pos = np.arange(first, first + n)
    slots = [16 * pages[p // 16] + p % 16 for p in pos]
    d, out = qkv.to(dev), torch.empty((n, 16, 128), dtype=BF16, device=dev)
    ints = [torch.tensor(list(x), dtype=torch.int32, device=dev) for x in (pos, slots)]
    rt.rope_append(D.make_dims(16, hkv), rope, pool, *ints, d[:, :16], d[:, 16:16 + hkv],
                   d[:, 16 + hkv:], out)
    new = [ow.rotate(qkv[:, 16:16 + hkv].float().numpy(), rope.table.cpu().numpy(), pos),
           qkv[:, 16 + hkv:].float().numpy()]
    for i, (b, rows, slot) in enumerate([(pages[0], slice(0, 5), 11), (pages[1], slice(5, 9), 0)]):
        for x, name in enumerate("kv"):
            got = getattr(pool, name)[b].cpu().numpy()
            got = got.swapaxes(1, 2)[:, SWAP] if name == "v" else got
            for h in range(hkv):
                want, e = ow.append_page(codes[x, i, h], exps[x, i, h],
                                         new[x][rows, h].astype(np.float64), slot)
                assert np.array_equal(got[h], want), (name, i, h)
                assert int(getattr(pool, name + "_exp")[b, h]) == e


# q_len, kv_len, window, sinks
NORMS = [([1] * 40, [1000 + 7 * i for i in range(40)], None, 0), ([1] * 9, [4000] * 9, 1500, 20),
         ([1] * 600, [1100] * 600, None, 0), ([90], [1100], None, 0), ([200, 40], [1300, 1000], 900, 7),
         ([40, 1, 1], [1500, 1200, 1300], None, 0)]


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("case", range(len(NORMS)))
def test_rows_in_the_two_norm(dev, ws, case, kv8):
    """Heads of rows over about a thousand keys: the error in the 2-norm.

    A rounding to bf16 is within 2^-8 of a value, 2^-8 / sqrt(3) in the mean square; with bf16
    output that is the output's, and, of a prompt, as much again from its weights (each
    key's part of the output has its own, and the parts add up in squares as the outputs
    do).  Twice 128 of them together stay within 1.3 of their mean (5 standard deviations of a
    sum of squares).  Scores of products of codes are within 2^-15 of sum |q k|, 11 here at
    most, which moves a weight by 2^-11.5.  fp32 output: 2^-15 for all.  A key left out is
    2^-5 of a row over a thousand."""
    q_len, kv_len, window, sinks = NORMS[case]
    m = Mix(dev, 8, 2, q_len, kv_len, window, sinks, kv8, seed=case)
    for dtype in (BF16, FP32):
        got = m.run(ws, dtype, SCALE).double().cpu().numpy()
        at = 0
        for s, (ql, kl) in enumerate(zip(q_len, kv_len)):
            pick = np.unique(np.linspace(0, ql - 1, 12).astype(int))
            if ql == 1 and s % max(1, len(q_len) // 20):
                at += 1
                continue
            k, v = (np.nan_to_num(x) for x in (m.k[s], m.v[s]))
            want = ow.attention_rows(m.q[s][pick], k, v, SCALE, kl - ql + pick, window, sinks)
            err = np.linalg.norm(got[at + pick] - want, axis=2) / np.linalg.norm(want, axis=2)
            if dtype is FP32:
                bound = 2.0 ** -15
            else:
                bound = 1.3 * 2.0 ** -8 / 3 ** 0.5 * (2 if ql > 1 else 1) ** 0.5
                bound += 2.0 ** -11.5 if kv8 else 0.0
            assert (err <= bound).all(), float((err / bound).max())
            at += ql


# hq, hkv, q_len, kv_len, window, sinks, tuning: tiles of 128 rows, of few, whole and split,
# without a window, with one, with sinks.
PARTLY = [
    (8, 2, 100, 400, None, 0, (0, 0, 0, 32)), (8, 2, 100, 400, 90, 0, (0, 0, 0, 32)),
    (2, 2, 300, 300, None, 0, (0, 0, 0, 128)), (2, 2, 300, 700, 40, 37, (0, 128, 0, 100)),
    (16, 2, 50, 200, 33, 5, (0, 64, 0, 16)), (8, 2, 40, 400, 70, 0, (0, 0, 0, 8)),
    (2, 2, 90, 200, 21, 18, (0, 64, 0, 32)), (4, 2, 64, 64, None, 0, (0, 0, 0, 1)),
]


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("case", range(len(PARTLY)))
def test_values_that_some_rows_of_a_prompt_see(dev, ws, case, dtype, kv8):
    """A NaN or infinite value reaches its dim of the rows that see its key and no other
    output, be the others' tokens earlier or later in the same tile."""
    hq, hkv, ql, kl, window, sinks, tn = PARTLY[case]
    m = Mix(dev, hq, hkv, [ql], [kl], window, sinks, kv8, seed=case)
    batch, g = m.batch(D.dlfp_tuning(*tn)), hq // hkv
    plain = m.run(ws, dtype, SCALE, batch=batch)
    pos = np.arange(kl - ql, kl)
    kept = m.pool.v.view(torch.uint8).clone()
    seen_by_some = np.flatnonzero(ow.sees(pos[:, None], np.arange(kl)[None], window, sinks).any(0))
    rng = np.random.default_rng(case)
    for turn in range(3):
        m.pool.v.view(torch.uint8).copy_(kept)
        hits = np.zeros((3, ql, hkv, 128), bool)       # of +inf, -inf, NaN
        for key in rng.choice(seen_by_some, size=6, replace=False):
            head, dim, kind = rng.integers(hkv), rng.integers(128), 2 if kv8 else rng.integers(3)
            page = m.pool.v.view(torch.uint8) if kv8 else m.pool.v
            page[int(m.table[0, key // 16]), head, dim, SWAP[key % 16]] = \
                0xFF if kv8 else (math.inf, -math.inf, math.nan)[kind]
            hits[kind, ow.sees(pos, key, window, sinks), head, dim] = True
        hits = [torch.from_numpy(np.repeat(h, g, axis=1)).to(dev) for h in hits]
        want = plain.clone()
        want[hits[0]] = math.inf
        want[hits[1]] = -math.inf
        want[hits[2] | (hits[0] & hits[1])] = math.nan
        got = m.run(ws, dtype, SCALE, batch=batch)
        wrong = ~((got == want) | (got.isnan() & want.isnan()))
        where = wrong.nonzero()[:4].tolist()
        assert not where
    assert D.dlfp_workspace_error(ws.buf) == 0


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("tn", [(0, 0, 0, 32), (0, 64, 0, 32), (0, 64, 0, 4)])
def test_rows_that_are_not_numbers_beside_infinite_values(dev, ws, tn, dtype):
    """A NaN query's row stays NaN where a value that it sees is infinite, and changes no
    other row; a NaN key those of the rows that see it."""
    ql, kl = 100, 400
    m = Mix(dev, 8, 2, [ql], [kl], None, 0, False, seed=3)
    batch = m.batch(D.dlfp_tuning(*tn))
    want = m.run(ws, dtype, SCALE, batch=batch)

    def put(page, key, head, dim, x):
        at = (key % 16, dim) if page is m.pool.k else (dim, SWAP[key % 16])
        page[(int(m.table[0, key // 16]), head, *at)] = x
    put(m.pool.v, 340, 0, 5, math.inf)
    put(m.pool.v, 100, 1, 7, -math.inf)
    put(m.pool.k, 370, 1, 9, math.nan)
    m.dq[60, 1, 3] = math.nan                           # its token at 360
    want[40:, :4, 5] = math.inf
    want[:, 4:, 7] = -math.inf
    want[60, 1] = math.nan
    want[70:, 4:] = math.nan
    got = m.run(ws, dtype, SCALE, batch=batch)
    wrong = ~((got == want) | (got.isnan() & want.isnan()))
    where = wrong.nonzero()[:4].tolist()
    assert not where


@pytest.mark.parametrize("kv8", [False, True])
def test_batches_without_sequences(dev, ws, kv8):
    """Nothing to do: nothing is launched, and a later call finds the workspace as it was."""
    dims = D.make_dims(8, 2)
    pool = rt.KVPool8(3, 2, dev) if kv8 else rt.KVPool(3, 2, dev, 0)
    batch = rt.WindowBatch(dims, [], [], np.zeros((0, 2), np.int32), 3, dev, 16, 2)
    q, k = (torch.empty((0, h, 128), dtype=BF16, device=dev) for h in (8, 2))
    batch.append(rt.Rope(4, dev), pool, q, k, k, q)
    batch.attention(pool, q, SCALE, q, ws)
    m = Mix(dev, 8, 2, [20, 1], [200, 77], 40, 3, kv8)
    m.check(m.run(ws, BF16, SCALE, D.dlfp_tuning(64, 64)), SCALE)
    assert D.dlfp_workspace_error(ws.buf) == 0


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("q_len,kv_len,tn", [
    ([1, 1, 1], [700, 33, 1500], None), ([1, 1, 1], [700, 33, 1500], (128,)),
    ([1] * 70, [40 + i for i in range(70)], None), ([100, 1], [300, 200], (0, 0, 0, 16)),
    ([100, 20], [300, 200], (0, 64, 0, 8)), ([1] * 300 + [1500], [100] * 300 + [1500], None)])
def test_queries_that_are_not_finite(dev, ws, q_len, kv_len, tn, dtype, kv8):
    """A row's head whose query holds a NaN or an infinity is NaN, every other as it was."""
    m = Mix(dev, 16, 2, q_len, kv_len, None, 0, kv8, seed=9)
    batch = m.batch(D.dlfp_tuning(*tn) if tn else None)
    want = m.run(ws, dtype, SCALE, batch=batch)
    n = sum(q_len)
    for row, head, dim, x in ((0, 3, 7, math.nan), (n // 2, 9, 100, math.inf), (n - 1, 15, 0, -math.inf),
                              (n - 1, 8, 127, math.nan)):
        m.dq[row, head, dim] = x
        want[row, head] = math.nan
    got = m.run(ws, dtype, SCALE, batch=batch)
    wrong = ~((got == want) | (got.isnan() & want.isnan()))
    where = wrong.nonzero()[:4].tolist()
    assert not where
    assert D.dlfp_workspace_error(ws.buf) == 0
