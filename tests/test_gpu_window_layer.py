"""GPU: the rotating append and the attention that reads its pages, as a serving program runs them.

Several iterations of a small server against an oracle that keeps its own cache,
captured graphs, other streams, far pages, and the replay over 8-bit windowed
layers.
"""
import math
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from _paged_mixes import Mix, bf16
from oracle import window as ow
from paper_2609_38386_amd import dlfp as D
from paper_2609_38386_amd import replay as rp
from paper_2609_38386_amd import runtime as rt

pytestmark = pytest.mark.gpu
SCALE = 1.0 / math.sqrt(128)
SWAP = [(t & 3) | ((t & 4) << 1) | ((t & 8) >> 1) for t in range(16)]


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available()
    D.lib()
    return torch.device("cuda:0")


@pytest.fixture(scope="module")
def ws(dev):
    return rt.Workspace(dev, 16 << 20)


class Server:
    """Sequences over one pool of pages; new tokens come from one generator."""

    def __init__(self, dev, hq, hkv, kv8, window, sinks, rotary, blocks=64):
        self.dev, self.hq, self.hkv, self.kv8 = dev, hq, hkv, kv8
        self.window, self.sinks = window, sinks
        self.dims = D.make_dims(hq, hkv)
        self.rope = rt.Rope(600, dev, theta=1e4, rotary_dim=rotary)
        self.pool = rt.KVPool8(blocks, hkv, dev) if kv8 else rt.KVPool(blocks, hkv, dev, 0x7FC0)
        self.free = list(np.random.default_rng(1).permutation(blocks))
        self.rng = np.random.default_rng(2)
        self.pages, self.k, self.v = {}, {}, {}   # the oracle's cache: dequantised rows
        self.state = {}                           # 8-bit pages: (codes, byte) per page and head

    def step(self, work, spread=1.0):
        """One iteration: {sequence: new tokens}; returns (output, what the oracle needs)."""
        names = list(work)
        q_len = [work[s] for s in names]
        total = sum(q_len)
        new = bf16(self.rng.normal(size=(total, self.hq + 2 * self.hkv, 128)) * spread)
        kv_len = []
        for s, n in zip(names, q_len):
            have = len(self.k.get(s, ()))
            pages = self.pages.setdefault(s, [])
            while 16 * len(pages) < have + n:
                pages.append(int(self.free.pop()))
            kv_len.append(have + n)
        table = np.full((len(names), max(len(self.pages[s]) for s in names)), -1, np.int32)
        for i, s in enumerate(names):
            table[i, :len(self.pages[s])] = self.pages[s]
        batch = rt.WindowBatch(self.dims, q_len, kv_len, table, self.pool.num_blocks, self.dev,
                               self.window, self.sinks)
        d = new.to(self.dev)
        q, k, v = d[:, :self.hq], d[:, self.hq:self.hq + self.hkv], d[:, self.hq + self.hkv:]
        turned = torch.empty((total, self.hq, 128), dtype=torch.bfloat16, device=self.dev)
        batch.append(self.rope, self.pool, q, k, v, turned)
        at, queries = 0, []
        for s, n, kl in zip(names, q_len, kv_len):
            pos = np.arange(kl - n, kl)
            rows = new[at:at + n].float().numpy()
            t = ow.rotate(rows[:, :self.hq + self.hkv], self.rope.table.cpu().numpy(), pos)
            queries.append(bf16(t[:, :self.hq]).double().numpy())
            self._append(s, kl - n, t[:, self.hq:], rows[:, self.hq + self.hkv:])
            at += n
        info = SimpleNamespace(q_len=q_len, kv_len=kv_len, q=queries, k=[self.k[s] for s in names],
                               v=[self.v[s] for s in names], hq=self.hq, hkv=self.hkv,
                               window=self.window, sinks=self.sinks, kv8=self.kv8, v_exp=-4)
        return batch, turned, info

    def _append(self, s, first, k, v):
        for name, x in (("k", k), ("v", v)):
            have = getattr(self, name).get(s, np.zeros((0, self.hkv, 128)))
            if not self.kv8:
                x = bf16(x).double().numpy()
                getattr(self, name)[s] = np.concatenate([have, x])
                continue
            rows = np.concatenate([have, np.zeros(x.shape)])
            done = 0
            while done < len(x):
                p, o = (first + done) // 16, (first + done) % 16
                n = min(16 - o, len(x) - done)
                for h in range(self.hkv):
                    codes, e = self.state.get((s, name, p, h), (np.zeros((16, 128), np.uint8), 127))
                    codes, e = ow.append_page(codes, e, x[done:done + n, h].astype(np.float64), o)
                    self.state[s, name, p, h] = codes, e
                    rows[16 * p:16 * p + o + n, h] = ow.E4M3[codes[:o + n]] * 2.0 ** (e - 127)
                done += n
            getattr(self, name)[s] = rows


@pytest.mark.parametrize("kv8", [False, True])
@pytest.mark.parametrize("window,sinks", [(None, 0), (24, 3), (64, 20)])
def test_iterations_of_a_server(dev, ws, kv8, window, sinks):
    """Chunked prompts beside decoders; every iteration's rows against the oracle's cache."""
    s = Server(dev, 8, 2, kv8, window, sinks, 64 if window else 128)
    plan = [{"a": 33}, {"b": 5, "a": 20}, {"c": 70, "a": 1, "b": 1}, {"c": 1, "a": 1, "b": 17},
            {"d": 2, "a": 1, "b": 1, "c": 1}] + [{"a": 1, "b": 1, "c": 1, "d": 1}] * 4
    for i, work in enumerate(plan):
        batch, q, info = s.step(work, spread=1.0 + 0.2 * i)   # later tokens raise the exponents
        for dtype in (torch.bfloat16, torch.float32):
            out = torch.full((batch.num_tokens + 2, 8, 128), 7.0, dtype=dtype, device=dev)
            batch.attention(s.pool, q, SCALE, out[:batch.num_tokens], ws)
            Mix.check(info, out[:batch.num_tokens], SCALE)
            assert (out[batch.num_tokens:] == 7.0).all()
    if kv8:   # the pages themselves
        for (seq, name, p, h), (codes, e) in s.state.items():
            b = s.pages[seq][p]
            got = getattr(s.pool, name).view(torch.uint8)[b, h].cpu().numpy()
            got = got.T[SWAP] if name == "v" else got
            n = min(16, len(s.k[seq]) - 16 * p)
            assert np.array_equal(got[:n], codes[:n])
            assert int(getattr(s.pool, name + "_exp")[b, h]) == e
    assert D.dlfp_workspace_error(ws.buf) == 0


@pytest.mark.parametrize("kv8", [False, True])
def test_captured_and_replayed(dev, kv8):
    """Append and attention in graphs that share a workspace, replayed in turn with eager
    work between; every replay gives the eager bits."""
    mixes = [Mix(dev, 8, 2, [40, 1, 1, 1], [300, 900, 64, 33], 100, 5, kv8, seed=1),
             Mix(dev, 8, 2, [1, 1], [2000, 777], None, 0, kv8, seed=2)]
    ws = rt.Workspace(dev, 16 << 20)
    rope = rt.Rope(2100, dev)
    runs = []
    for m in mixes:
        b = m.batch(D.dlfp_tuning(256, 128))
        assert b.meta.num_groups > 0
        g = torch.Generator(device=dev).manual_seed(5)
        qkv = torch.empty((b.num_tokens, 12, 128), dtype=torch.bfloat16, device=dev).normal_(generator=g)
        turned = torch.empty_like(m.dq)
        out = torch.empty_like(m.dq)

        def call(m=m, b=b, qkv=qkv, turned=turned, out=out):
            b.append(rope, m.pool, qkv[:, :8], qkv[:, 8:10], qkv[:, 10:], turned)
            b.attention(m.pool, turned, SCALE, out, ws)
        call()
        torch.cuda.synchronize()
        runs.append((call, out, out.clone(), turned, turned.clone()))
    graphs = []
    for call, *_ in runs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append(graph)
    for turn in range(4):
        for graph, (call, out, want, turned, want_q) in zip(graphs, runs):
            out.fill_(float("nan"))
            turned.fill_(float("nan"))
            graph.replay()
            if turn == 2:
                torch.cuda.synchronize()
            assert torch.equal(out.view(torch.int16), want.view(torch.int16))
            assert torch.equal(turned.view(torch.int16), want_q.view(torch.int16))
        runs[turn % 2][0]()
    assert D.dlfp_workspace_error(ws.buf) == 0


@pytest.mark.parametrize("kv8", [False, True])
def test_other_streams_and_repeats(dev, ws, kv8):
    """Two streams with a workspace each, calls that overlap; all give the same bits."""
    m = Mix(dev, 16, 2, [30, 1, 1], [700, 1500, 90], 512, 9, kv8, seed=3)
    b = m.batch(D.dlfp_tuning(128, 128))
    want = m.run(ws, torch.bfloat16, SCALE, batch=b)
    m.check(want, SCALE)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    spaces = [rt.Workspace(dev, 16 << 20, s) for s in streams]
    outs = [[torch.full_like(want, float("nan")) for _ in range(6)] for _ in streams]
    torch.cuda.synchronize()
    for i in range(6):
        for s, space, o in zip(streams, spaces, outs):
            b.attention(m.pool, m.dq, SCALE, o[i], space, stream=s)
    with torch.cuda.stream(streams[0]):   # the current stream when none is given
        extra = torch.full_like(want, float("nan"))
        b.attention(m.pool, m.dq, SCALE, extra, spaces[0])
    torch.cuda.synchronize()
    for o in [extra] + outs[0] + outs[1]:
        assert torch.equal(o.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("kv8", [False, True])
def test_far_pages(dev, ws, kv8):
    """Pages whose byte offsets pass 32 bits."""
    first = (1 << 32) // (2 * (2048 if kv8 else 4096)) + 3
    m = Mix(dev, 16, 2, [20, 1, 1], [300, 500, 3], 128, 4, kv8, seed=4, first_block=first)
    for dtype in (torch.bfloat16, torch.float32):
        m.check(m.run(ws, dtype, SCALE), SCALE)


@pytest.mark.parametrize("kv8", [False, True])
def test_long_context_and_large_scores(dev, ws, kv8):
    """20000 keys over many splits; queries that leave one key most of the weight."""
    m = Mix(dev, 8, 1, [1, 1, 3], [20000, 4097, 4500], None, 0, kv8, seed=5)
    for dtype in (torch.bfloat16, torch.float32):
        m.check(m.run(ws, dtype, SCALE), SCALE)
    m = Mix(dev, 8, 1, [1, 1, 40], [3000, 65, 600], 500, 33, kv8, seed=6, spread=40.0)
    for dtype in (torch.bfloat16, torch.float32):
        m.check(m.run(ws, dtype, SCALE), SCALE)


@pytest.mark.parametrize("kv8", [False, True])
def test_values_that_are_not_numbers(dev, ws, kv8):
    """A decoder that sees a NaN value has NaN in that dim alone, a NaN key makes its row
    NaN, an infinite value is that infinity; what it does not see changes nothing."""
    m = Mix(dev, 4, 1, [1, 1, 1], [100, 100, 100], 40, 2, kv8, seed=7)
    want = m.run(ws, torch.bfloat16, SCALE)
    m.check(want, SCALE)
    nan = 0x7F if kv8 else float("nan")

    def put(s, key, name, dim, x):
        b = int(m.table[s, key // 16])
        page = getattr(m.pool, name)
        page = page.view(torch.uint8) if kv8 else page
        if name == "k":
            page[b, 0, key % 16, dim] = x
        else:
            page[b, 0, dim, SWAP[key % 16]] = x
    put(0, 70, "v", 9, nan)
    put(1, 1, "k", 3, nan)
    if not kv8:
        put(2, 99, "v", 5, -math.inf)
    got = m.run(ws, torch.bfloat16, SCALE)
    assert got[0, :, 9].isnan().all() and not got[0, :, :9].isnan().any()
    assert not got[0, :, 10:].isnan().any() and got[1].isnan().all()
    if not kv8:
        assert (got[2, :, 5] == -math.inf).all()
        got[2, :, 5] = want[2, :, 5]
    assert torch.equal(got[2], want[2])


@pytest.mark.parametrize("kv8", [False, True])
def test_block_ids_outside_the_pool(dev, kv8):
    """Met on the device: the launch raises the workspace error word and reads block 0."""
    m = Mix(dev, 8, 2, [40, 1], [300, 900], None, 0, kv8, seed=8)
    space = rt.Workspace(dev, 16 << 20)
    for row, bad in ((0, m.blocks), (1, -1)):
        b = m.batch()
        b.d_block_table[row, 3] = bad
        out = torch.empty_like(m.dq)
        b.attention(m.pool, m.dq, SCALE, out, space)
        assert D.dlfp_workspace_error(space.buf) == 1
        D.dlfp_workspace_init(space.buf)
    m.check(m.run(space, torch.bfloat16, SCALE), SCALE)


@pytest.mark.parametrize("bits,window,rotary", [(8, None, True), (8, 512, True), (16, 256, False)])
def test_replay(dev, bits, window, rotary):
    """The closed loop over such layers: every token produced, the controller fed."""
    cfg = rp.ReplayConfig(seed=802, n_requests=8, rate_per_s=400.0, prompt_hi=1024, out_len=12,
                          kv_bits=bits, window=window, sinks=4 if window else 0, rotary=rotary)
    ex = rp.GpuExecutor(cfg, dev)
    trace = []
    got = rp.run_replay(cfg, rp.Policy(rp.Policy.DLFP, target_ms=0.05, cfg=cfg), ex, trace=trace)
    assert got["reconciled"] and got["guarded_iterations"] > 0
    assert all(0.0 < it["layer_ms"] < 50.0 for it in trace)
    assert torch.isfinite(ex.out[:4].float()).all()
    assert D.dlfp_workspace_error(ex.ws.buf) == 0


def test_tensors_of_another_device_than_the_current_one(dev, ws, monkeypatch):
    m = Mix(dev, 4, 2, [1], [20], None, 0, False)
    batch, out = m.batch(), torch.empty(m.dq.shape, dtype=torch.bfloat16, device=dev)
    rope = rt.Rope(32, dev)
    at = torch.zeros(1, dtype=torch.int32, device=dev)
    k = torch.zeros(1, 2, 128, dtype=torch.bfloat16, device=dev)
    monkeypatch.setattr(D, "_current_device", lambda: dev.index + 1)
    with pytest.raises(ValueError, match="current device"):
        batch.attention(m.pool, m.dq, SCALE, out, ws)
    with pytest.raises(ValueError, match="current device"):
        rt.rope_append(m.dims, rope, m.pool, at, at, m.dq, k, k, torch.empty_like(m.dq))


@pytest.mark.parametrize("window,sinks", [(None, 0), (300, 20)])
def test_value_pages_of_far_scales(dev, ws, window, sinks):
    """Value scales up to 2^140 apart beside scores that leave either kind of page all of
    a row's weight."""
    m = Mix(dev, 16, 2, [1, 1, 1, 9], [1000, 700, 333, 200], window, sinks, True, seed=6,
            spread=60.0, v_exps=[-100, -40, 40])
    for dtype in (torch.bfloat16, torch.float32):
        for tn in (None, D.dlfp_tuning(64)):
            m.check(m.run(ws, dtype, SCALE, tn), SCALE)


def test_pool_of_other_heads(dev, ws):
    m = Mix(dev, 4, 2, [1], [20], None, 0, False)
    pool = rt.KVPool(4, 1, dev)
    with pytest.raises(ValueError, match="heads"):
        m.batch().attention(pool, m.dq, SCALE, torch.empty_like(m.dq), ws)
    at = torch.zeros(1, dtype=torch.int32, device=dev)
    k = torch.zeros(1, 2, 128, dtype=torch.bfloat16, device=dev)
    with pytest.raises(ValueError, match="heads"):
        rt.rope_append(m.dims, rt.Rope(4, dev), pool, at, at, m.dq, k, k, torch.empty_like(m.dq))


def test_staged_batch_over_its_capacity(dev):
    stage = rt.WindowStagedBatch(D.make_dims(4, 2), 2, 8, 64, dev, 16, 2)
    table = np.arange(4, dtype=np.int32).reshape(2, 2)
    lens = [np.array(x, np.int32) for x in ([7, 2], [7, 20])]
    with pytest.raises(D.DlfpError):
        stage.build(*lens, table, 4)
    stage.build(np.array([6, 2], np.int32), np.array([7, 20], np.int32), table, 4)
    torch.cuda.synchronize()
    assert stage.d_positions.tolist() == [1, 2, 3, 4, 5, 6, 18, 19]
    assert stage.d_slots.tolist() == [1, 2, 3, 4, 5, 6, 50, 51]


def test_parts_on_the_host(dev):
    """A rope or a pool of which a part is on the host is refused."""
    dims, at = D.make_dims(4, 2), torch.zeros(1, dtype=torch.int32, device=dev)
    k = torch.zeros(1, 2, 128, dtype=torch.bfloat16, device=dev)
    q = torch.zeros(1, 4, 128, dtype=torch.bfloat16, device=dev)
    pool = rt.KVPool8(2, 2, dev)
    with pytest.raises(ValueError, match="another device"):
        rt.rope_append(dims, rt.Rope.of(torch.zeros(4, 128)), pool, at, at, q, k, k, q.clone())
    with pytest.raises(ValueError):
        rt.KVPool8.of(pool.k, pool.v.cpu(), pool.k_exp, pool.v_exp)
    with pytest.raises(ValueError):
        rt.KVPool8.of(pool.k, pool.v, pool.k_exp.cpu(), pool.v_exp)
