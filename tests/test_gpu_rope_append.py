"""GPU: the rotating appends against the oracle, bit for bit.

Keys and queries are turned in fp32 with every product and sum rounded, so the
oracle in fp32 (numpy rounds each operation) gives the same bits; bf16 and e4m3
codes are then rounded once.  Every slot that is not written has to keep its
bits.
"""
import numpy as np
import pytest
import torch

from _paged_mixes import bf16
from oracle import window as ow
from paper_2609_38386_amd import dlfp as D
from paper_2609_38386_amd import runtime as rt

pytestmark = pytest.mark.gpu
SWAP = [(t & 3) | ((t & 4) << 1) | ((t & 8) >> 1) for t in range(16)]


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available()
    D.lib()
    return torch.device("cuda:0")


def _same(x, y):
    """Equal bits; a NaN has many patterns, any of which will do."""
    bits = [torch.where(t.isnan(), torch.full_like(t, float("nan")), t).view(torch.int16)
            for t in (x.cpu(), y.cpu())]
    return torch.equal(*bits)


class Append:
    """Sequences of new tokens, their pages and every input, on the host and the device."""

    def __init__(self, dev, hq, hkv, seqs, seed=0, rotary=128, interleaved=False, positions=None,
                 values=None):
        rng = np.random.default_rng(seed)
        self.dev, self.hq, self.hkv = dev, hq, hkv
        self.dims = D.make_dims(hq, hkv)
        q_len, kv_len = np.array([a for a, _ in seqs]), np.array([b for _, b in seqs])
        seq = np.repeat(np.arange(len(seqs)), q_len)
        self.pos = np.concatenate([np.arange(n - p, n) for p, n in seqs]).astype(np.int32)
        self.n = len(self.pos)
        pages = [(s, p) for s, (ql, n) in enumerate(seqs)
                 for p in range((n - ql) // 16, -(-n // 16))]
        self.blocks = len(pages) + 4
        ids = dict(zip(pages, rng.permutation(self.blocks)))
        self.slots = np.array([ids[s, p // 16] * 16 + p % 16 for s, p in zip(seq, self.pos)],
                              np.int32)
        self.rope = rt.Rope(positions or int(kv_len.max()), dev, theta=1e4, rotary_dim=rotary,
                            interleaved=interleaved)
        self.interleaved = interleaved
        x = rng.normal(size=(self.n, hq + 2 * hkv, 128)) if values is None else values(rng, self)
        self.qkv = bf16(x)
        self.dqkv = self.qkv.to(dev)

    def parts(self, x):
        return x[:, :self.hq], x[:, self.hq:self.hq + self.hkv], x[:, self.hq + self.hkv:]

    def turned(self, x):
        ok = (self.pos >= 0) & (self.pos < self.rope.table.size(0))
        with np.errstate(all="ignore"):
            return ow.rotate(x.float().numpy(), self.rope.table.cpu().numpy(),
                             np.where(ok, self.pos, 0), self.interleaved)

    def ints(self):
        return (torch.from_numpy(self.pos).to(self.dev), torch.from_numpy(self.slots).to(self.dev))

    def call(self, pool, q_out):
        q, k, v = self.parts(self.dqkv)
        rt.rope_append(self.dims, self.rope, pool, *self.ints(), q, k, v, q_out)

    def check_queries(self, q_out, before):
        want = bf16(self.turned(self.parts(self.qkv)[0]))
        ok = torch.from_numpy((self.pos >= 0) & (self.pos < self.rope.table.size(0)))
        want = torch.where(ok[:, None, None], want, before.cpu())
        assert _same(q_out, want)

    def written(self):
        """(token, block, slot) of the tokens that go into the pool."""
        for t, (p, s) in enumerate(zip(self.pos, self.slots)):
            if 0 <= p < self.rope.table.size(0) and 0 <= s < 16 * self.blocks:
                yield t, s // 16, s % 16


SEQS = [
    [(1, 1)], [(1, 16), (1, 17), (1, 300)], [(16, 16)], [(16, 32)], [(5, 70)], [(40, 41)],
    [(1, 5), (35, 100), (1, 64), (3, 18), (17, 17)], [(130, 133), (1, 2)], [(1, 1 + i) for i in range(37)],
]
SHAPES = [(16, 8), (8, 8), (8, 1), (64, 8), (2, 2)]


def _poison_pool(a, kv8, rng):
    shape = (a.blocks, a.hkv)
    if kv8:
        codes = [rng.integers(0, 255, size=(*shape, *x)).astype(np.uint8) for x in ((16, 128), (128, 16))]
        exps = [rng.integers(100, 126, size=shape).astype(np.uint8) for _ in range(2)]
        t = [torch.from_numpy(x).to(a.dev) for x in codes + exps]
        return rt.KVPool8.of(t[0].view(torch.float8_e4m3fn), t[1].view(torch.float8_e4m3fn), *t[2:])
    pool = rt.KVPool(a.blocks, a.hkv, a.dev)
    for x in (pool.k, pool.v):
        x.copy_(bf16(rng.normal(size=tuple(x.shape))))
    return pool


def _check_bf16(a, pool, before):
    k = bf16(a.turned(a.parts(a.qkv)[1]))
    v = a.parts(a.qkv)[2]
    want_k, want_v = (x.clone() for x in before)
    for t, b, s in a.written():
        want_k[b, :, s] = k[t]
        want_v[b, :, :, SWAP[s]] = v[t]
    assert _same(pool.k, want_k)
    assert _same(pool.v, want_v)


def _runs(a):
    runs = []
    for t, b, s in a.written():
        if runs and runs[-1][0] + runs[-1][3] == t and runs[-1][1] == b and \
                runs[-1][2] + runs[-1][3] == s:
            runs[-1][3] += 1
        else:
            runs.append([t, b, s, 1])
    return runs


def _check_kv8(a, pool, before):
    new = [a.turned(a.parts(a.qkv)[1]).astype(np.float64), a.parts(a.qkv)[2].double().numpy()]
    want = [x.copy() for x in before]
    want[1] = np.ascontiguousarray(want[1].transpose(0, 1, 3, 2)[:, :, SWAP])   # token rows
    for t, b, s, n in _runs(a):
        for x in range(2):
            for h in range(a.hkv):
                want[x][b, h], want[2 + x][b, h] = ow.append_page(
                    want[x][b, h], want[2 + x][b, h], new[x][t:t + n, h], s)
    got = [x.view(torch.uint8).cpu().numpy() for x in (pool.k, pool.v, pool.k_exp, pool.v_exp)]
    got[1] = got[1].transpose(0, 1, 3, 2)[:, :, SWAP]
    for name, g, w in zip(("k_exp", "v_exp", "k", "v"), got[2:] + got[:2], want[2:] + want[:2]):
        if name in "kv":   # a NaN has two codes
            g, w = (np.where((x & 127) == 127, 127, x) for x in (g, w))
        assert np.array_equal(g, w), (name, np.argwhere(g != w)[:5])


def _run(a, kv8, seed=3):
    rng = np.random.default_rng(seed)
    pool = _poison_pool(a, kv8, rng)
    if kv8:
        before = [x.view(torch.uint8).cpu().numpy().copy() for x in (pool.k, pool.v, pool.k_exp, pool.v_exp)]
    else:
        before = [pool.k.cpu(), pool.v.cpu()]
    q_out = torch.full((a.n, a.hq, 128), 7.0, dtype=torch.bfloat16, device=a.dev)
    was = q_out.clone()
    a.call(pool, q_out)
    torch.cuda.synchronize()
    a.check_queries(q_out, was)
    (_check_kv8 if kv8 else _check_bf16)(a, pool, before)
    return pool


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("seqs", range(len(SEQS)))
def test_append(dev, seqs, kv8):
    hq, hkv = SHAPES[seqs % len(SHAPES)]
    _run(Append(dev, hq, hkv, SEQS[seqs], seed=seqs), kv8)


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rotary", [32, 64, 128])
def test_rotations(dev, rotary, interleaved, kv8):
    _run(Append(dev, 16, 8, SEQS[6], 1, rotary, interleaved), kv8)


@pytest.mark.parametrize("kv8", [False, True])
def test_tokens_left_out(dev, kv8):
    """Slots outside the pool: the query is turned, nothing written; positions outside the
    table: nothing at all."""
    a = Append(dev, 16, 8, [(20, 40), (1, 9), (1, 10), (30, 30)], positions=33)
    a.slots[[3, 20]] = [-1, a.blocks * 16]
    a.pos[21] = -1                       # and the positions 33 .. 39 of the first sequence
    _run(a, kv8)


def _hard(rng, a):
    x = rng.normal(size=(a.n, a.hq + 2 * a.hkv, 128))
    x *= 2.0 ** rng.integers(-40, 20, size=(a.n, a.hq + 2 * a.hkv, 1))
    x[0] = 0.0
    x[1, :, ::3] = np.inf
    x[2, :, 5] = np.nan
    x[3] = -np.inf
    x[4] *= 1e-30
    x[5] = np.where(rng.random(x[5].shape) < 0.5, 448.0, -449.0)
    x[6] = 2.0 ** -126
    x[7] = 1e30
    return x


@pytest.mark.parametrize("kv8", [False, True])
def test_hard_values(dev, kv8):
    _run(Append(dev, 16, 8, [(1, 5), (1, 16), (1, 17), (1, 3), (1, 40), (1, 90), (1, 1), (1, 33), (40, 45)],
                seed=2, values=_hard), kv8)


def test_a_page_token_by_token(dev):
    """A page filled one token at a time, its exponents growing on the way, gives what the
    oracle gives step by step; a full page's tokens keep their values."""
    rng = np.random.default_rng(0)
    dims, rope = D.make_dims(8, 4), rt.Rope(64, dev)
    pool = rt.KVPool8(3, 4, dev)
    want = [np.zeros((4, 16, 128), np.uint8) for _ in "kv"]
    exps = np.full((2, 4), 127)
    for t in range(16):
        x = bf16(rng.normal(size=(1, 16, 128)) * 2.0 ** rng.integers(-6, 6))
        d = x.to(dev)
        out = torch.empty((1, 8, 128), dtype=torch.bfloat16, device=dev)
        at = torch.tensor([t], dtype=torch.int32, device=dev)
        rt.rope_append(dims, rope, pool, at, at + 16, d[:, :8], d[:, 8:12], d[:, 12:], out)
        new = [ow.rotate(x[:, 8:12].float().numpy(), rope.table.cpu().numpy(), [t]), x[:, 12:].float().numpy()]
        for i in range(2):
            for h in range(4):
                want[i][h], exps[i, h] = ow.append_page(want[i][h], exps[i, h], new[i][:, h], t)
        assert np.array_equal(pool.k.view(torch.uint8)[1].cpu().numpy(), want[0])
        got = pool.v.view(torch.uint8)[1].cpu().numpy().transpose(0, 2, 1)[:, SWAP]
        assert np.array_equal(got, want[1])
        assert np.array_equal(torch.stack([pool.k_exp[1], pool.v_exp[1]]).cpu().numpy(), exps)
    assert int(pool.k.view(torch.uint8)[[0, 2]].max()) == 0


@pytest.mark.parametrize("kv8", [False, True])
def test_in_place_and_repeated(dev, kv8):
    """Queries turned in place inside the projection's rows; a second call with the same
    tokens leaves the pages as they are."""
    a = Append(dev, 16, 8, SEQS[6], seed=9)
    pool = _run(a, kv8)
    first = [x.clone() for x in vars(pool).values() if isinstance(x, torch.Tensor)]
    qkv = a.dqkv.clone()
    q, k, v = a.parts(qkv)
    rt.rope_append(a.dims, a.rope, pool, *a.ints(), q, k, v, q)
    torch.cuda.synchronize()
    a.check_queries(q.contiguous(), q)
    assert torch.equal(qkv[:, 16:].view(torch.int16), a.dqkv[:, 16:].view(torch.int16))
    for x, y in zip(first, [x for x in vars(pool).values() if isinstance(x, torch.Tensor)]):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


@pytest.mark.parametrize("kv8", [False, True])
def test_far_rows_and_pages(dev, kv8):
    """Token rows and pages whose offsets pass 32 bits."""
    hkv, n, ld = 8, 3, (1 << 30) + 8
    blocks = (1 << 32) // (hkv * 2048) + 50 if kv8 else (1 << 32) // (hkv * 4096) + 50
    a = Append(dev, 16, hkv, [(3, 35)], seed=4)
    buf = torch.empty(((n - 1) * ld + 32 * 128,), dtype=torch.bfloat16, device=dev)
    rows = buf.as_strided((n, 32, 128), (ld, 128, 1))
    rows.copy_(a.dqkv)
    q, k, v = rows[:, :16], rows[:, 16:24], rows[:, 24:]
    if kv8:
        def empty(*x):
            return torch.empty(x, dtype=torch.uint8, device=dev)
        pool = rt.KVPool8.of(empty(blocks, hkv, 16, 128), empty(blocks, hkv, 128, 16),
                             empty(blocks, hkv), empty(blocks, hkv))
    else:
        pool = rt.KVPool(blocks, hkv, dev)
    b = blocks - 1
    slots = torch.tensor([b * 16, b * 16 + 1, b * 16 + 2], dtype=torch.int32, device=dev)
    out = torch.empty((n, 16, 128), dtype=torch.bfloat16, device=dev)
    rt.rope_append(a.dims, a.rope, pool, a.ints()[0], slots, q, k, v, out)
    torch.cuda.synchronize()
    a.check_queries(out, out)
    new = a.turned(a.parts(a.qkv)[1])
    if kv8:
        for h in range(hkv):
            want, e = ow.append_page(np.zeros((16, 128), np.uint8), 0, new[:, h].astype(np.float64), 0)
            assert np.array_equal(pool.k[b, h, :3].cpu().numpy(), want[:3]) and int(pool.k_exp[b, h]) == e
    else:
        assert torch.equal(pool.k[b, :, :3].cpu(), bf16(new).transpose(0, 1))
        assert torch.equal(pool.v[b, :, :, :3].cpu(), a.parts(a.qkv)[2].permute(1, 2, 0))


@pytest.mark.parametrize("kv8", [False, True])
def test_no_tokens(dev, kv8):
    pool = rt.KVPool8(2, 8, dev) if kv8 else rt.KVPool(2, 8, dev, fill_bits=0)
    none = torch.empty((0, 16, 128), dtype=torch.bfloat16, device=dev)
    at = torch.empty(0, dtype=torch.int32, device=dev)
    rt.rope_append(D.make_dims(16, 8), rt.Rope(4, dev), pool, at, at, none, none[:, :8],
                   none[:, :8], none)


LONG = [
    [(1, 1 + 7 * i % 50) for i in range(521)] + [(90, 300)],
    [(517, 1003)] + [(1, 1 + 5 * i % 40) for i in range(19)] + [(3, 33), (20, 30)],
    [(1100, 1100)], [(2, 2 + 5 * i % 40) for i in range(300)],
]


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("left_out", [False, True])
@pytest.mark.parametrize("seqs", range(len(LONG)))
def test_many_tokens(dev, seqs, left_out, kv8):
    """More tokens than the launches for few take; with slots outside the pool, the runs of
    a page that a token left out makes two of."""
    a = Append(dev, 4, 2, LONG[seqs], seed=seqs)
    if left_out:
        a.slots[np.arange(5, a.n, 37)] = -1
    _run(a, kv8)
