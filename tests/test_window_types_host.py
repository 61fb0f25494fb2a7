"""Types that the calls of dlfp_cache.h would read as others are refused (no GPU needed)."""
from types import SimpleNamespace

import numpy as np
import pytest
import torch

from paper_2609_38386_amd import dlfp as D
from paper_2609_38386_amd import runtime as rt

DIMS = D.make_dims(16, 8)


def _append(pool, q=torch.bfloat16, k=torch.bfloat16, v=torch.bfloat16, out=torch.bfloat16,
            at=torch.int32, slots=torch.int32, rope=None):
    rt.rope_append(DIMS, rope or rt.Rope(10, "cpu"), pool, torch.zeros(3, dtype=at),
                   torch.zeros(3, dtype=slots), torch.zeros((3, 16, 128), dtype=q),
                   torch.zeros((3, 8, 128), dtype=k), torch.zeros((3, 8, 128), dtype=v),
                   torch.zeros((3, 16, 128), dtype=out))


@pytest.mark.parametrize("pool", [rt.KVPool8(4, 8, "cpu"), rt.KVPool(4, 8, "cpu")])
def test_appends(pool):
    with pytest.raises(ValueError, match="on a device"):   # all types right, on the host
        _append(pool)
    for name in ("q", "k", "v", "out"):
        for bad in (torch.float16, torch.int16, torch.uint16, torch.float32):
            with pytest.raises(ValueError, match="bf16"):
                _append(pool, **{name: bad})
    for name in ("at", "slots"):
        for bad in (torch.float32, torch.uint32, torch.int64):
            with pytest.raises(ValueError, match="int32"):
                _append(pool, **{name: bad})


def test_rope_tables():
    rt.Rope.of(torch.zeros(4, 128))
    for bad in (torch.int32, torch.float64, torch.bfloat16):
        with pytest.raises(ValueError, match="float32"):
            rt.Rope.of(torch.zeros((4, 128), dtype=bad))


def test_attention():
    pool = rt.KVPool(1, 8, "cpu")
    batch = rt.WindowBatch(DIMS, [3], [3], np.zeros((1, 1), np.int32), 1, "cpu")
    ws = SimpleNamespace(ensure=lambda *a: torch.zeros(1 << 20, dtype=torch.uint8))

    def call(pool=pool, q=torch.bfloat16, out=torch.bfloat16):
        batch.attention(pool, torch.zeros((3, 16, 128), dtype=q), 0.1,
                        torch.zeros((3, 16, 128), dtype=out), ws)
    for p in (pool, rt.KVPool8(1, 8, "cpu")):
        with pytest.raises(ValueError, match="on a device"):
            call(p)
        for bad in (torch.float16, torch.int16):
            with pytest.raises(ValueError, match="bf16"):
                call(p, q=bad)
    for name in ("d_work", "d_block_table"):
        kept = getattr(batch, name)
        for bad in (torch.float32, torch.int64):
            setattr(batch, name, kept.to(bad))
            with pytest.raises(ValueError, match="int32"):
                call()
        setattr(batch, name, kept)


def test_pools():
    pool = rt.KVPool8(4, 8, "cpu")
    parts = (pool.k, pool.v, pool.k_exp, pool.v_exp)
    rt.KVPool8.of(*parts)
    rt.KVPool8.of(pool.k.view(torch.uint8), pool.v.view(torch.uint8), *parts[2:])   # the codes
    for bad in (torch.float8_e4m3fnuz, torch.float8_e5m2, torch.int8, torch.bool):
        for i in range(2):
            x = list(parts)
            x[i] = x[i].view(torch.uint8).view(bad)
            with pytest.raises(ValueError, match="e4m3"):
                rt.KVPool8.of(*x)


@pytest.mark.parametrize("window,sinks", [(2 ** 31, 0), (2 ** 32 + 5, 0), (5, 2 ** 32 + 1), (5, 2 ** 31),
                                          (-2 ** 32 + 1, 0)])
def test_windows_past_32_bits(window, sinks):
    """Not the number that 32 bits keep of them."""
    for batch in (lambda: rt.WindowBatch(DIMS, [1], [60], np.zeros((1, 4), np.int32), 1, "cpu", window,
                                         sinks),
                  lambda: rt.WindowStagedBatch(DIMS, 1, 1, 8, "cpu", window, sinks)):
        with pytest.raises(ValueError, match="32 bits"):
            batch()
    rt.WindowBatch(DIMS, [1], [60], np.zeros((1, 4), np.int32), 1, "cpu", 2 ** 31 - 1, 2 ** 31 - 1)


def test_lists_and_tables_shorter_than_the_metadata():
    """A work list or block table that does not hold what the metadata counts."""
    pool = rt.KVPool(4, 8, "cpu")
    batch = rt.WindowBatch(DIMS, [3, 1], [3, 40], np.arange(6, dtype=np.int32).reshape(2, 3) % 4, 4, "cpu")
    ws = SimpleNamespace(ensure=lambda *a: torch.zeros(1 << 20, dtype=torch.uint8))
    q = torch.zeros((4, 16, 128), dtype=torch.bfloat16)
    for name, short in (("d_work", batch.d_work[:-1]), ("d_block_table", batch.d_block_table[:1]),
                        ("d_work", batch.d_work[::2])):
        kept = getattr(batch, name)
        setattr(batch, name, short)
        with pytest.raises(ValueError, match="metadata|contiguous"):
            batch.attention(pool, q, 0.1, q.clone(), ws)
        setattr(batch, name, kept)


def test_exponents_of_the_binding():
    """The calls under a pool's take its four tensors apart."""
    pool = rt.KVPool8(4, 8, "cpu")
    q, k = torch.zeros((3, 16, 128), dtype=torch.bfloat16), torch.zeros((3, 8, 128), dtype=torch.bfloat16)
    at = torch.zeros(3, dtype=torch.int32)
    meta = rt.WindowBatch(DIMS, [3], [3], np.zeros((1, 1), np.int32), 4, "cpu")
    for bad in (pool.k_exp[:3], pool.k_exp[:, :7], pool.k_exp.to(torch.int32), pool.k_exp.t()):
        for exps in ((bad, pool.v_exp), (pool.k_exp, bad)):
            with pytest.raises(ValueError, match="exponents"):
                D.dlfp_rope_append_kv8(DIMS, rt.Rope(4, "cpu").c, at, at, q, k, k, q, pool.k, pool.v, *exps)
            with pytest.raises(ValueError, match="exponents"):
                D.dlfp_attention_kv8(DIMS, meta.meta, meta.d_work, meta.d_block_table, q, pool.k,
                                     pool.v, *exps, 0.1, q.clone(), torch.zeros(1 << 20, dtype=torch.uint8))
