"""Performance cases of the rotating cache append and of windowed and 8-bit attention.

Each case is one call that a serving program makes for a layer of one mixed
continuous-batching iteration:

- kind "append": queries and keys are rotated to their positions, keys and
  values go into their pages, of bf16 or of 8 bits with an exponent for each
  page and KV head (`dlfp_rope_append`, `dlfp_rope_append_kv8`);
- kind "attention": `decoders` sequences of one new token with contexts spread
  over [ctx_lo, ctx_hi] beside `prompts` prompts of about `chunk` new tokens
  over about `prefix` cached ones, over bf16 pages (`dlfp_attention_window`) or
  8-bit pages (`dlfp_attention_kv8`).  With `window` > 0 a row sees the last
  `window` keys up to its own and the sequence's first `sinks`; with 0 every
  key up to its own.

Head counts and batches are those of the Qwen3-0.6B / 8B / 32B attention layers
(head_dim 128, 8 KV heads, 16 / 32 / 64 query heads) that the chunk-size sweeps
run.  Queries, keys and values are N(0, 1); pages are a random permutation of
the pool, and pages that no row sees are not in the block table (-1).  The
lengths are fixed by the case; the seed decides their order, the pages and the
values.
"""
import math

import numpy as np
import torch

own = False

HEAD_DIM = 128
PAGE = 16
SCALE = 1.0 / math.sqrt(HEAD_DIM)
THETA = 1.0e6
CODE_MAX = 448.0                   # largest e4m3 value
EXP_MIN, EXP_BIAS = -100, 127      # least exponent of a page, and what its byte adds
E4M3 = torch.float8_e4m3fn
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
# Position of token slot t inside a value page row (slots 4-7 and 8-11 trade places).
VALUE_POS = [(t & 3) | ((t & 4) << 1) | ((t & 8) >> 1) for t in range(PAGE)]


def _append(hq, decoders, ctx_lo, ctx_hi, chunk, prefix, cache, rotary=128, interleaved=False,
            hkv=8):
    return {"kind": "append", "hq": hq, "hkv": hkv, "decoders": decoders, "ctx_lo": ctx_lo,
            "ctx_hi": ctx_hi, "prompts": 1 if chunk else 0, "chunk": chunk, "prefix": prefix,
            "cache": cache, "rotary": rotary, "interleaved": interleaved}


def _attention(hq, decoders, ctx_lo, ctx_hi, chunk, prefix, cache, window=0, sinks=0, prompts=None,
               out="bf16", hkv=8):
    return {"kind": "attention", "hq": hq, "hkv": hkv, "decoders": decoders, "ctx_lo": ctx_lo,
            "ctx_hi": ctx_hi, "prompts": (1 if chunk else 0) if prompts is None else prompts,
            "chunk": chunk, "prefix": prefix, "cache": cache, "window": window, "sinks": sinks,
            "out": out}


def listed():
    return [
        # A nearly idle server's layer: four decoders, bound by the launch and its round trips.
        {"name": "append-few", **_append(16, 4, 64, 256, 0, 0, "bf16")},
        # An uncapped Qwen3-0.6B chunk that starts inside a page.
        {"name": "append-chunk", **_append(16, 0, 0, 0, 2048, 4099, "bf16")},
        # Qwen3-32B decoders, each into its own partly filled 8-bit page.
        {"name": "append-kv8-decode", **_append(64, 256, 2048, 32768, 0, 0, "e4m3")},
        # A batch at the 8192-token budget into 8-bit pages beside 64 decoders.
        {"name": "append-kv8-mixed", **_append(32, 64, 1024, 8192, 8128, 1001, "e4m3")},
        # The smallest windowed batch, fp32 output.
        {"name": "window-few", **_attention(16, 4, 64, 256, 0, 0, "bf16", 128, 4, out="fp32")},
        # Qwen3-0.6B, a capped chunk beside its decoders, in a 1024-key window.
        {"name": "window-mixed", **_attention(16, 32, 512, 2048, 256, 3840, "bf16", 1024, 4)},
        # Qwen3-32B long-context decoders in a 4096-key window.
        {"name": "window-decode", **_attention(64, 256, 2048, 32768, 0, 0, "bf16", 4096, 4)},
        # Qwen3-32B prompt chunk in a window whose edges lie inside tiles.
        {"name": "window-chunk", **_attention(64, 0, 0, 0, 4096, 8192, "bf16", 4000, 5)},
        # Qwen3-8B decoders over 8-bit pages.
        {"name": "kv8-decode", **_attention(32, 128, 1024, 8192, 0, 0, "e4m3")},
        # Few rows over very long contexts: only splitting the keys fills the chip.
        {"name": "kv8-long", **_attention(64, 3, 60000, 130000, 0, 0, "e4m3", out="fp32")},
        # Qwen3-8B prompts of odd lengths alone.
        {"name": "kv8-chunk", **_attention(32, 0, 0, 0, 1999, 6145, "e4m3", prompts=2)},
        # Qwen3-8B at its operating point, windowed, 8-bit pages.
        {"name": "kv8-mixed", **_attention(32, 128, 1024, 8192, 1999, 7777, "e4m3", 2048, 16)},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    hq = rng.choice([16, 32, 64])
    hkv = 8 if rng.random() < 0.85 else 16
    cache = rng.choice(["bf16", "e4m3"])
    share = rng.choice(["mixed", "decode", "prompt"])
    decoders = 0 if share == "prompt" else _log_int(rng, 1, 256)
    lo = _log_int(rng, 1, 32768)
    if rng.random() < 0.35:
        chunk = 0 if share == "decode" else _log_int(rng, 2, 7900)
        return _append(hq, decoders, lo, 4 * lo, chunk, rng.randint(0, 8192), cache,
                       rotary=rng.choice([128, 128, 64, 32]), interleaved=rng.random() < 0.25,
                       hkv=hkv)
    window = rng.choice([0, _log_int(rng, 1, 8192)])
    sinks = rng.choice([0, rng.randint(1, 64)]) if window else 0
    # At most about 600k visible decode keys of 8 heads.
    most = 600_000 * 8 // (hkv * max(decoders, 1))
    window = min(window, max(1, most - 64))
    lo = lo if window else max(1, min(lo, most // 4))
    chunk = 0 if share == "decode" else _log_int(rng, 2, 4096)
    prompts = rng.choice([1, 1, 2, 3]) if chunk else 0
    # At most a third of the largest listed prompt's pairs in the padded plain form.
    room = 700_000_000 // (hq * max(chunk * prompts, 1))
    chunk = min(chunk, max(2, room))
    prefix = rng.randint(0, max(0, min(16384, room - chunk)))
    return _attention(hq, decoders, lo, 4 * lo, chunk, prefix if chunk else 0, cache, window, sinks,
                      prompts=prompts, out=rng.choice(["bf16", "bf16", "fp32"]), hkv=hkv)


# ----------------------------------------------------------------- inputs

def _device():
    return torch.device("cuda:0" if torch.cuda.is_available() else "cpu")


def _generator(seed, salt=0):
    return torch.Generator(device=_device()).manual_seed(1000003 * int(seed) + salt)


def _lengths(case):
    """(q_len, kv_len) of the packed batch, prompts first; kv_len counts the new tokens."""
    n, lo, hi = case["decoders"], case["ctx_lo"], case["ctx_hi"]
    prompts = [(max(1, case["chunk"] - 7 * i), max(0, case["prefix"] - 301 * i))
               for i in range(case["prompts"])]
    q_len = [p for p, _ in prompts] + [1] * n
    kv_len = [p + c for p, c in prompts]
    kv_len += [max(1, int(lo + (hi - lo) * (i + 0.5) / n)) for i in range(n)]
    return np.array(q_len, np.int64), np.array(kv_len, np.int64)


def _spans(case):
    """Per sequence: pages with visible sink keys, then the first and the end of its other pages."""
    q_len, kv_len = _lengths(case)
    window, sinks = case.get("window", 0), case.get("sinks", 0)
    end = -(-kv_len // PAGE)
    if case["kind"] == "append":
        return 0 * end, (kv_len - q_len) // PAGE, end
    if not window:
        return 0 * end, 0 * end, end
    sink = np.minimum(-(-np.minimum(sinks, kv_len) // PAGE), end)
    first = np.maximum(kv_len - q_len + 1 - window, 0) // PAGE
    return sink, np.maximum(first, sink), end


def _table(case, seed):
    """(order of the sequences, block table, blocks of the pool): pages in sight only."""
    q_len, kv_len = _lengths(case)
    sink, first, end = _spans(case)
    rng = np.random.default_rng(int(seed))
    order = np.concatenate([np.arange(case["prompts"]),
                            case["prompts"] + rng.permutation(case["decoders"])]).astype(np.int64)
    q_len, kv_len, sink, first, end = (x[order] for x in (q_len, kv_len, sink, first, end))
    page = np.arange(int(end.max()))[None, :]
    seen = (page < sink[:, None]) | ((page >= first[:, None]) & (page < end[:, None]))
    blocks = int(seen.sum())
    table = np.full(seen.shape, -1, np.int32)
    table[seen] = rng.permutation(blocks).astype(np.int32)
    return q_len, kv_len, table, blocks


def _pool(case, blocks, seed):
    """The cache: what earlier calls have written into its pages."""
    gen, dev = _generator(seed, 7919), _device()
    shapes = {"k": (blocks, case["hkv"], PAGE, HEAD_DIM), "v": (blocks, case["hkv"], HEAD_DIM, PAGE)}
    pool = {}
    for name, shape in shapes.items():
        if case["cache"] == "bf16":
            pool[name] = torch.empty(shape, dtype=torch.bfloat16, device=dev).normal_(generator=gen)
            continue
        exps = torch.randint(-9, -6, shape[:2], generator=gen, device=dev)
        codes = torch.empty(shape, dtype=torch.bfloat16, device=dev).normal_(generator=gen)
        codes *= torch.exp2(-exps.to(torch.bfloat16))[..., None, None]
        pool[name] = codes.clamp_(-CODE_MAX, CODE_MAX).to(E4M3)
        pool[name + "_exp"] = (exps + EXP_BIAS).to(torch.uint8)
    return pool


def _new_tokens(case, seed, tokens):
    """Queries, keys and values of the new tokens, as one projection leaves them."""
    hq, hkv = case["hq"], case["hkv"]
    qkv = torch.empty((tokens, hq + 2 * hkv, HEAD_DIM), dtype=torch.bfloat16, device=_device())
    qkv.normal_(generator=_generator(seed))
    return qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]


def _rope_table(case, positions):
    """[positions][rotary]: cosines, then sines, of a pair's angles, from 64 bits."""
    r = case["rotary"]
    freq = THETA ** (-2.0 * torch.arange(r // 2, dtype=torch.float64, device=_device()) / r)
    angle = torch.arange(positions, dtype=torch.float64, device=_device())[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def _packed(case, q_len, kv_len, table):
    """Positions and flat cache slots of the new tokens, in packed order."""
    seq = np.repeat(np.arange(len(q_len)), q_len)
    row = np.arange(len(seq)) - np.repeat(np.cumsum(q_len) - q_len, q_len)
    pos = (kv_len - q_len)[seq] + row
    return pos, table[seq, pos // PAGE].astype(np.int64) * PAGE + pos % PAGE


def prepare(case, seed):
    dev = _device()
    q_len, kv_len, table, blocks = _table(case, seed)
    tokens = int(q_len.sum())
    s = {"case": case, "pool": _pool(case, blocks, seed), "q_len": q_len, "kv_len": kv_len}
    q, k, v = _new_tokens(case, seed, tokens)
    if case["kind"] == "append":
        s.update(q=q, k=k, v=v, q_out=torch.empty(q.shape, dtype=q.dtype, device=dev))
        s["table"] = _rope_table(case, int(kv_len.max()))
        pos, slots = _packed(case, q_len, kv_len, table)
        s["positions"] = torch.from_numpy(pos.astype(np.int32)).to(dev)
        s["slots"] = torch.from_numpy(slots.astype(np.int32)).to(dev)
    else:
        s["q"] = q.contiguous()
        s["block_table"] = torch.from_numpy(table).to(dev)
        sink, first, end = (int(x.max()) for x in _spans(case))
        s["sink_pages"] = sink
        s["out"] = torch.empty(q.shape, dtype=DTYPES[case["out"]], device=dev)
    if own:
        from paper_2609_38386_amd import dlfp, runtime
        dims = dlfp.make_dims(case["hq"], case["hkv"])
        s["dims"], p = dims, s["pool"]
        if case["cache"] == "bf16":
            s["pages"] = runtime.KVPool.of(p["k"], p["v"])
        else:
            s["pages"] = runtime.KVPool8.of(p["k"], p["v"], p["k_exp"], p["v_exp"])
        if case["kind"] == "append":
            s["rope"] = runtime.Rope.of(s["table"], interleaved=case["interleaved"])
        else:
            s["workspace"] = runtime.Workspace(dev, 16 << 20)
            s["batch"] = runtime.WindowBatch(dims, q_len, kv_len, table, blocks, dev,
                                             window=case["window"] or None, sinks=case["sinks"])
    return s


# ----------------------------------------------------------------- the calls

def run(state):
    s, case = state, state["case"]
    p = s["pool"]
    if case["kind"] == "append":
        if own:
            from paper_2609_38386_amd import runtime
            runtime.rope_append(s["dims"], s["rope"], s["pages"], s["positions"], s["slots"],
                                s["q"], s["k"], s["v"], s["q_out"])
        else:
            _plain_append(s)
        return [s["q_out"]] + [p[x] for x in ("k", "v", "k_exp", "v_exp") if x in p]
    if own:
        s["batch"].attention(s["pages"], s["q"], SCALE, s["out"], s["workspace"])
        return [s["out"]]
    return [_plain_attention(s)]


# ----------------------------------------------------------------- plain forms

def _rotate(x, table, positions, interleaved):
    """x: [T][heads][128] -> its first table.shape[1] dims turned by the position's angles, fp32."""
    r = table.shape[1]
    row = table[positions.long()][:, None]
    c, s = row[..., :r // 2], row[..., r // 2:]
    x = x.float()
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    y = (a * c - b * s, b * c + a * s)
    y = torch.stack(y, -1).flatten(-2) if interleaved else torch.cat(y, -1)
    return torch.cat([y, x[..., r:]], -1)


def _plain_append(s):
    case, p = s["case"], s["pool"]
    s["q_out"].copy_(_rotate(s["q"], s["table"], s["positions"], case["interleaved"]))
    k = _rotate(s["k"], s["table"], s["positions"], case["interleaved"])
    v = s["v"].float()
    slots = s["slots"].long()
    block, slot = slots // PAGE, slots % PAGE
    place = (slot & 3) | ((slot & 4) << 1) | ((slot & 8) >> 1)
    if case["cache"] == "bf16":
        p["k"][block, :, slot] = k.to(torch.bfloat16)
        p["v"][block, :, :, place] = v.to(torch.bfloat16)
        return
    # The pages written, with the first slot that the call writes of each: the
    # slots before it hold older tokens, which follow a page's larger exponent.
    start = torch.full((p["k"].shape[0],), PAGE, device=slots.device)
    start = start.scatter_reduce(0, block, slot, "amin")
    page = block[slot == start[block]]
    old = torch.arange(PAGE, device=slots.device)[None] < start[page][:, None]
    swap = torch.tensor(VALUE_POS, device=slots.device)
    _quantize(p["k"], p["k_exp"], k, block, page, start, old[:, None, :, None], (block, slot), True)
    _quantize(p["v"], p["v_exp"], v, block, page, start, old[:, swap][:, None, None], (block, place),
              False)


def _quantize(codes, exps, x, block, page, start, old, at, rows):
    """Writes x ([T][hkv][128], fp32) into 8-bit pages: codes and exponents."""
    amax = torch.zeros(exps.shape, device=x.device)
    most = torch.where(x.isfinite(), x.abs(), 0.0).amax(-1)
    amax = amax.scatter_reduce(0, block[:, None].expand_as(most), most, "amax")[page]
    mantissa, power = torch.frexp(amax)            # amax = mantissa 2^power, mantissa in [1/2, 1)
    need = torch.where(mantissa <= 0.875, power - 9, power - 8)   # 448 = 0.875 * 2^9
    need = torch.where(amax > 0, need, EXP_MIN).clamp(min=EXP_MIN)
    was = exps[page].int() - EXP_BIAS
    now = torch.where((start[page] > 0)[:, None], torch.maximum(need, was), need)
    codes = codes.view(torch.uint8)
    kept = codes[page].view(E4M3).float()
    moved = kept * torch.exp2((was - now).float())[..., None, None]
    codes[page] = torch.where(old, moved, kept).to(E4M3).view(torch.uint8)
    exps[page] = (now + EXP_BIAS).to(torch.uint8)
    new = torch.ldexp(x, -(exps[block].int() - EXP_BIAS)[..., None])
    new = torch.where(new.isfinite(), new, math.nan).to(E4M3).view(torch.uint8)
    if rows:
        codes[at[0], :, at[1]] = new
    else:
        codes[at[0], :, :, at[1]] = new


def _plain_attention(s):
    """Prompts and decoders each as one padded batch."""
    case, n = s["case"], s["case"]["prompts"]
    split = int(s["q_len"][:n].sum())
    out = torch.empty(s["q"].shape, dtype=DTYPES[case["out"]], device=s["q"].device)
    if n:
        _padded(s, slice(0, n), s["q"][:split], out[:split])
    if case["decoders"]:
        _padded(s, slice(n, None), s["q"][split:], out[split:])
    return out


def _padded(s, which, q, out):
    case, p, dev = s["case"], s["pool"], q.device
    hkv, window, sinks = case["hkv"], case["window"] or 1 << 40, case["sinks"]
    g = case["hq"] // hkv
    q_np, kv_np, table = s["q_len"][which], s["kv_len"][which], s["block_table"][which].long()
    # The pages in sight: the first ones, then those from the first row's window on.
    first_np = np.maximum(kv_np - q_np + 1 - window, 0) // PAGE
    width = int((-(-kv_np // PAGE) - first_np).max())
    q_len, kv_len, first = (torch.from_numpy(x).to(dev) for x in (q_np, kv_np, first_np))
    sink = torch.arange(s["sink_pages"], device=dev).expand(len(q_np), -1)
    rest = first[:, None] + torch.arange(width, device=dev)
    twice = torch.cat([torch.zeros_like(sink), rest < s["sink_pages"]], 1).bool()
    pages = torch.cat([sink, rest], 1)
    block = table.gather(1, pages.clamp(max=table.shape[1] - 1)).clamp(min=0)
    key = (pages[..., None] * PAGE + torch.arange(PAGE, device=dev)).flatten(1)
    here = (key < kv_len[:, None]) & ~twice.repeat_interleave(PAGE, 1)

    def gathered(name):
        # [B][pages][hkv][16][128], values [128][16]
        if name + "_exp" in p:
            x = p[name].view(torch.uint8)[block].view(E4M3).float()
            x *= torch.exp2(p[name + "_exp"][block].float() - EXP_BIAS)[..., None, None]
        else:
            x = p[name][block].float()
        x = x if name == "k" else x[..., VALUE_POS].transpose(-1, -2)
        return x.transpose(1, 2).flatten(2, 3)             # [B][hkv][keys][128]

    # The rows of each sequence, padded to the longest.
    most, begin = int(q_np.max()), torch.cumsum(q_len, 0) - q_len
    row = torch.arange(most, device=dev)
    valid = row < q_len[:, None]
    at = begin[:, None] + torch.minimum(row, q_len[:, None] - 1)
    pos = (kv_len - q_len)[:, None] + row
    x = q.float()[at].unflatten(2, (hkv, g)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    back = pos[:, :, None] - key[:, None, :]               # [B][rows][keys]
    seen = here[:, None] & (back >= 0) & ((back < window) | (key < sinks)[:, None])
    score = torch.matmul(x, gathered("k").transpose(-1, -2)).mul_(SCALE).unflatten(2, (most, g))
    score.masked_fill_(~seen[:, None, :, None], -math.inf)
    score -= score.amax(-1, keepdim=True)
    weight = score.exp_()
    total = weight.sum(-1, keepdim=True)
    value = gathered("v").masked_fill_(~seen.any(1)[:, None, :, None], 0.0)
    y = torch.matmul(weight.flatten(2, 3), value).unflatten(2, (most, g)) / total
    out.copy_(y.permute(0, 2, 1, 3, 4).flatten(2, 3)[valid].to(out.dtype))


# ----------------------------------------------------------------- work and exact results

def work(case):
    q_len, kv_len = _lengths(case)
    tokens, hq, hkv = int(q_len.sum()), case["hq"], case["hkv"]
    kv_token = hkv * HEAD_DIM * 2 * (2 if case["cache"] == "bf16" else 1)
    if case["kind"] == "append":
        data = tokens * (4 * hq * HEAD_DIM + 4 * hkv * HEAD_DIM + kv_token + 4 * case["rotary"])
        return {"bytes": data, "flops": 6 * tokens * (hq + hkv) * case["rotary"] // 2}
    window, sinks = case["window"] or 1 << 40, case["sinks"]

    def pairs(q, n):
        pos = np.arange(n - q, n)
        return int(np.minimum(pos + 1, np.minimum(pos + 1, window) +
                              np.minimum(sinks, np.maximum(pos + 1 - window, 0))).sum())

    keys = 0
    for q, n in zip(q_len, kv_len):
        lo = max(n - q + 1 - window, 0)
        keys += int(n - lo + min(sinks, lo))
    flops = 4 * HEAD_DIM * hq * sum(pairs(q, n) for q, n in zip(q_len, kv_len))
    rows = tokens * hq * HEAD_DIM * (2 + (4 if case["out"] == "fp32" else 2))
    return {"bytes": keys * kv_token + rows, "flops": flops}


def exact(case, seed):
    q_len, kv_len, table, blocks = _table(case, seed)
    pool = _pool(case, blocks, seed)
    q, k, v = _new_tokens(case, seed, int(q_len.sum()))
    if case["kind"] == "append":
        return _exact_append(case, q_len, kv_len, table, pool, q, k, v)
    return [_exact_attention(case, q_len, kv_len, table, pool, q.double())]


def _turned(x, table, pos, interleaved):
    """The rotation as a product with complex numbers."""
    r = table.shape[1]
    half = table[pos].double().unflatten(1, (2, r // 2))
    turn = torch.complex(half[:, 0], half[:, 1])[:, None]
    x = x.double().clone()
    if interleaved:
        z = torch.view_as_complex(x[..., :r].unflatten(-1, (r // 2, 2)).contiguous()) * turn
        x[..., :r] = torch.view_as_real(z).flatten(-2)
    else:
        z = torch.complex(x[..., :r // 2].contiguous(), x[..., r // 2:r].contiguous()) * turn
        x[..., :r] = torch.cat([z.real, z.imag], -1)
    return x


def _nearest_code(x):
    """The e4m3 value nearest to each of x (|x| <= 448), ties to even."""
    step = torch.exp2((torch.frexp(x)[1].clamp(min=-5) - 4).double())
    return torch.round(x / step) * step


def _exact_append(case, q_len, kv_len, table, pool, q, k, v):
    pos, slots = _packed(case, q_len, kv_len, table)
    dev = q.device
    turns, at = _rope_table(case, int(kv_len.max())), torch.from_numpy(pos).to(dev)
    q_out = _turned(q, turns, at, case["interleaved"])
    new = {"k": _turned(k, turns, at, case["interleaved"]), "v": v.double()}
    order = torch.tensor(VALUE_POS, device=dev)
    got = {}
    for name, x in new.items():
        codes = pool[name].double()
        codes = codes[..., order].transpose(-1, -2).contiguous() if name == "v" else codes
        block, slot = (torch.from_numpy(y).to(dev) for y in (slots // PAGE, slots % PAGE))
        if case["cache"] == "bf16":
            codes[block, :, slot] = x
        else:
            # Runs of new tokens inside a page, by their starts, a slot of the run at a time.
            starts = np.flatnonzero(np.r_[True, np.diff(slots) != 1] | (slots % PAGE == 0))
            length = np.diff(np.r_[starts, len(slots)])
            lead, length = (torch.from_numpy(y).to(dev) for y in (starts, length))
            page, begin = block[lead], slot[lead]
            amax = torch.zeros((len(starts), case["hkv"]), dtype=torch.float64, device=dev)
            for i in range(PAGE):
                inside = (i < length)[:, None]
                rows = x[(lead + i).clamp(max=len(slots) - 1)].abs().amax(-1)
                amax = torch.maximum(amax, torch.where(inside, rows, 0.0))
            need = torch.ceil(torch.log2(amax / CODE_MAX)).clamp(min=EXP_MIN)
            was = pool[name + "_exp"][page].double() - EXP_BIAS
            now = torch.where((begin > 0)[:, None], torch.maximum(need, was), need)
            exps = pool[name + "_exp"].double() - EXP_BIAS
            exps[page] = now
            for i in range(PAGE):
                kept = codes[page, :, i]
                moved = _nearest_code(kept * torch.exp2(was - now)[..., None])
                codes[page, :, i] = torch.where((i < begin)[:, None, None], moved, kept)
            codes[block, :, slot] = _nearest_code(x * torch.exp2(-exps[block])[..., None])
        got[name] = codes[..., order, :].transpose(-1, -2).contiguous() if name == "v" else codes
        if case["cache"] != "bf16":
            got[name + "_exp"] = None
    return [q_out] + [got[x] for x in ("k", "v", "k_exp", "v_exp") if x in got]


def _exact_attention(case, q_len, kv_len, table, pool, q):
    """Sequence by sequence, the keys of each row chosen by their positions."""
    hkv, window, sinks = case["hkv"], case["window"], case["sinks"]
    g, dev = case["hq"] // hkv, q.device
    out = torch.empty(q.shape, dtype=torch.float64, device=dev)
    row = 0
    for s in range(len(q_len)):
        p, n = int(q_len[s]), int(kv_len[s])
        lo = max(0, n - p + 1 - window) if window else 0
        keys = np.r_[np.arange(min(sinks, lo)), np.arange(lo, n)]
        used, inverse = np.unique(keys // PAGE, return_inverse=True)
        block = torch.from_numpy(table[s, used].astype(np.int64)).to(dev)
        pick = torch.from_numpy(inverse * PAGE + keys % PAGE).to(dev)
        kv = []
        for name in ("k", "v"):
            if name + "_exp" in pool:
                x = pool[name].view(torch.uint8)[block].view(E4M3).double()
                x = x * torch.exp2(pool[name + "_exp"][block].double() - EXP_BIAS)[..., None, None]
            else:
                x = pool[name][block].double()
            x = x.transpose(-1, -2)[..., VALUE_POS, :] if name == "v" else x
            kv.append(x.transpose(0, 1).flatten(1, 2)[:, pick].contiguous())
        key = torch.from_numpy(keys).to(dev)
        for h in range(hkv):
            kt = kv[0][h].t().contiguous()
            for t0 in range(0, p, 512):
                t1 = min(p, t0 + 512)
                pos = torch.arange(n - p + t0, n - p + t1, device=dev).repeat_interleave(g)[:, None]
                hidden = key[None] > pos
                if window:
                    hidden |= (key[None] <= pos - window) & (key[None] >= sinks)
                x = q[row + t0:row + t1, h * g:(h + 1) * g].reshape(-1, HEAD_DIM)
                score = (x @ kt * SCALE).masked_fill(hidden, -math.inf)
                y = torch.softmax(score, -1) @ kv[1][h]
                out[row + t0:row + t1, h * g:(h + 1) * g] = y.reshape(t1 - t0, g, HEAD_DIM)
        row += p
    return out
