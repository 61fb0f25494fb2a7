"""GPU: what the replay's layer proxy keeps on the device."""
import gc

import pytest
import torch

from paper_2609_38386_amd import replay as rp

pytestmark = pytest.mark.gpu

HIDDEN, MLP = 1024, 8192


def _kept(**fields):
    """Bytes that an executor holds, and its configuration."""
    cfg = rp.ReplayConfig(seed=3, n_requests=4, prompt_hi=1024, out_len=8, layer_proxy=True,
                          hidden=HIDDEN, mlp=MLP, **fields)
    gc.collect()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    ex = rp.GpuExecutor(cfg, torch.device("cuda:0"))
    torch.cuda.synchronize()
    gc.collect()
    kept = torch.cuda.memory_allocated() - before
    del ex
    return kept, cfg


@pytest.mark.parametrize("gated", [False, True])
def test_4_bit_weights_replace_the_bf16_ones(gated):
    """17/32 byte a weight instead of two; the allocator's steps of 512 bytes and 2 MiB aside."""
    wide, cfg = _kept(weight_bits=16, gated=gated)
    four, _ = _kept(weight_bits=4, gated=gated)
    heads = (2 * cfg.num_q_heads + 2 * cfg.num_kv_heads) * 128
    weights = HIDDEN * (heads + 3 * MLP)
    assert abs((wide - four) - weights * (2 - 17 / 32)) < 8 << 20


def test_gated_rows_are_as_wide_as_the_block():
    """The gated launch writes `mlp` columns a row, the plain one gate and up."""
    plain, cfg = _kept()
    gated, _ = _kept(gated=True)
    rows = cfg.budget + cfg.max_seqs
    assert abs((plain - gated) - rows * MLP * 2) < 8 << 20
