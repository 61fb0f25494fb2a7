"""GPU: 4-bit weights and the gated feed-forward projection against the float64 oracle.

Bounds are those of _projections.  Sizes are both sides of every block, wavefront step and
kernel: one token to a chunk, features down to 16, 64 columns to several thousand.
"""
import math

import numpy as np
import pytest
import torch

import _projections as pj
from oracle import ffn as of
from paper_2609_38386_amd import dlfp as D
from paper_2609_38386_amd import runtime as rt

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    assert torch.cuda.is_available()
    D.lib()
    return torch.device("cuda:0")


def _gen(dev, seed):
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    return g


def _bf16(dev, gen, shape, scale=1.0):
    x = torch.empty(shape, dtype=torch.float32, device=dev).normal_(generator=gen)
    return (x * scale).to(torch.bfloat16)


def _weights4(dev, gen, n, k):
    return rt.Weights4.of(*pj.random_codes(gen, n, k, device=dev))


def _values(w):
    return of.values(w.codes.cpu().numpy(), w.exps.cpu().numpy())


# ------------------------------------------------------------------- codes

@pytest.mark.parametrize("n,k,pad", [(1, 32, 0), (3, 96, 8), (17, 64, 40), (128, 1024, 0)])
def test_quantize_equals_the_oracle(dev, n, k, pad):
    gen = _gen(dev, n + k)
    wide = _bf16(dev, gen, (n, k + pad))
    wide *= torch.exp2(torch.randint(-40, 40, (n, 1), generator=gen, device=dev).float())
    w = rt.Weights4(n, k, dev)
    w.quantize(wide[:, :k])
    codes, exps = of.quantize(pj.f64(wide[:, :k]))
    assert np.array_equal(of.unpack(w.codes.cpu().numpy()), codes)
    assert np.array_equal(w.exps.cpu().numpy(), exps)
    back = torch.full((n, k + pad), 7.0, dtype=torch.bfloat16, device=dev)
    w.dequantize(back[:, :k])
    assert np.array_equal(pj.f64(back[:, :k]), _values(w))
    assert (back[:, k:] == 7.0).all()


def test_quantize_ties_signs_and_ends(dev):
    """Midpoints of neighbouring magnitudes, both zeros, largest magnitudes on both sides of an
    exponent's step, subnormal and largest bf16 values."""
    points = [0.0, -0.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.2490234375, 0.251953125, 4.9688,
              5.0313]
    rows = []
    for scale in (1.0, 2.0 ** -120, 2.0 ** 100, 2.0 ** -130):
        row = np.array((points + [-p for p in points] + [6.0] * 32)[:32]) * scale
        row[31] = 6.0 * scale
        rows.append(row)
    for most in (6.0, 6.03125, 7.96875, 4.03125, 3.0, 3.015625):
        rows.append(np.r_[most, -np.linspace(0, most, 31)])
    rows += [np.zeros(32), np.full(32, -0.0), np.r_[3.38e38, np.linspace(-3e38, 3e38, 31)],
             np.r_[1e-40, np.zeros(31)], np.full(32, 9.2e-41)]
    w = torch.from_numpy(np.array(rows)).to(torch.bfloat16).to(dev)
    got = rt.Weights4.from_bf16(w)
    codes, exps = of.quantize(pj.f64(w))
    assert np.array_equal(of.unpack(got.codes.cpu().numpy()), codes)
    assert np.array_equal(got.exps.cpu().numpy(), exps)


def test_a_group_with_a_value_that_is_not_finite(dev):
    w = torch.ones((2, 96), dtype=torch.bfloat16, device=dev)
    w[0, 5], w[1, 64], w[1, 70] = math.inf, math.nan, -math.inf
    got = rt.Weights4.from_bf16(w)
    assert got.exps.cpu().tolist() == [[255, 125, 125], [125, 125, 255]]
    back = torch.empty_like(w)
    got.dequantize(back)
    bad = torch.zeros((2, 96), dtype=torch.bool)
    bad[0, :32], bad[1, 64:] = True, True
    assert torch.equal(back.isnan().cpu(), bad) and (back.cpu()[~bad] == 1.0).all()


def test_every_code_in_every_scale(dev):
    codes = torch.arange(256, dtype=torch.uint8).repeat(256, 1).to(dev)   # [256][512 columns]
    exps = torch.arange(256, dtype=torch.uint8)[:, None].repeat(1, 16).to(dev)
    w = rt.Weights4.of(codes, exps)
    back = torch.empty((256, 512), dtype=torch.bfloat16, device=dev)
    w.dequantize(back)
    want = of.values(codes.cpu().numpy(), exps.cpu().numpy())
    want[np.abs(want) >= 2.0 ** 128] = np.inf * np.sign(want[np.abs(want) >= 2.0 ** 128])
    assert np.array_equal(pj.f64(back), want, equal_nan=True)


# ------------------------------------------------------------------- projections

SIZES = [(1, 16, 64), (1, 2048, 1024), (2, 48, 128), (5, 80, 192), (15, 1008, 320), (16, 32, 4160),
         (17, 64, 64), (31, 272, 1088), (33, 1024, 128), (63, 144, 576), (64, 64, 2048),
         (65, 16, 64), (100, 528, 448), (129, 256, 64), (200, 1040, 192), (257, 96, 512),
         (300, 2064, 128), (513, 304, 64), (777, 512, 1024), (1025, 272, 320), (256, 512, 8192),
         (40, 256, 16384), (3, 128, 16448), (130, 1040, 4160), (600, 336, 3136), (20, 4112, 576),
         (1100, 1040, 192)]


@pytest.mark.parametrize("m,n,k", SIZES)
def test_linear_w4(dev, m, n, k):
    """fp32 and bf16 output, 16-byte rows and rows that allow only 8-byte stores, x rows whole and
    apart; what lies between the rows of x is NaN, what lies around out stays."""
    gen = _gen(dev, m + 7 * n + 11 * k)
    w = _weights4(dev, gen, n, k)
    values = _values(w)
    for dtype, left, right, pad in ((torch.float32, 4, 4, 0), (torch.bfloat16, 8, 0, 8),
                                    (torch.bfloat16, 4, 8, 0)):
        wide = torch.full((m, k + pad), math.nan, dtype=torch.bfloat16, device=dev)
        x = wide[:, :k]
        x.copy_(_bf16(dev, gen, (m, k)))
        big = torch.full((m + 1, left + n + right), 7.0, dtype=dtype, device=dev)
        rt.linear(x, w, big[:m, left:left + n])
        torch.cuda.synchronize()
        pj.check(big[:m, left:left + n], *pj.linear(pj.f64(x), values, dtype))
        assert (big[:m, :left] == 7.0).all() and (big[:m, left + n:] == 7.0).all()
        assert (big[m] == 7.0).all()


def _some_sizes(seed):
    """Sizes over the whole range, their products bounded by what the oracle does quickly."""
    rng = np.random.default_rng(seed)
    k = 64 * int(round(2 ** rng.uniform(0, 8.6)))
    m = int(round(2 ** rng.uniform(0, 11.5)))
    most = max(1, int(4e8 / (m * k) / 16))
    return m, 16 * max(1, min(most, int(round(2 ** rng.uniform(0, 9))))), k


@pytest.mark.parametrize("seed", range(60))
def test_projections_of_some_sizes(dev, seed):
    """Both 4-bit calls and the bf16 one, with the workspace that the fastest form takes, one that
    is too small for it, and none; what the workspace held before is NaN."""
    m, n, k = _some_sizes(seed)
    gen = _gen(dev, seed)
    x = _bf16(dev, gen, (m, k))
    gate, up = _weights4(dev, gen, n, k), _weights4(dev, gen, n, k)
    g64, u64 = _values(gate), _values(up)
    x *= 1.5 / math.sqrt(float((g64 ** 2).sum(1).mean()))
    dense = [torch.empty((n, k), dtype=torch.bfloat16, device=dev) for _ in range(2)]
    for w, d in zip((gate, up), dense):
        w.dequantize(d)
    x64 = pj.f64(x)
    act = ("silu", "gelu")[seed % 2]
    plain, both = pj.linear(x64, g64, torch.float32), pj.gated(x64, g64, u64, act, torch.float32)
    out = torch.empty((m, n), dtype=torch.float32, device=dev)
    calls = ((D.LINEAR_W4, plain, lambda ws: rt.linear(x, gate, out, workspace=ws, stream=0)),
             (D.GATED_LINEAR_W4, both,
              lambda ws: rt.gated_linear(x, gate, up, out, act, workspace=ws, stream=0)),
             (D.GATED_LINEAR_BF16, both,
              lambda ws: rt.gated_linear(x, *dense, out, act, workspace=ws, stream=0)))
    for kind, want, call in calls:
        need = D.dlfp_projection_workspace(kind, m, n, k)
        for size in {need, need * 2 // 3 // 16 * 16, 0}:
            ws = None
            if size:
                room = torch.full((size // 4 + 64,), math.nan, dtype=torch.float32, device=dev)
                ws = room[:size // 4]
            out.fill_(math.nan)
            torch.cuda.synchronize()
            call(ws)
            torch.cuda.synchronize()
            pj.check(out, *want)
            assert not size or room[size // 4:].isnan().all()


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("m,n,k", SIZES)
def test_gated_linear(dev, four, m, n, k):
    gen = _gen(dev, 3 * m + 5 * n + 13 * k + four)
    if four:
        gate, up = _weights4(dev, gen, n, k), _weights4(dev, gen, n, k)
        g64, u64 = _values(gate), _values(up)
    else:
        gate, up = (_bf16(dev, gen, (n, k), 1.5 / math.sqrt(k)) for _ in range(2))
        g64, u64 = pj.f64(gate), pj.f64(up)
    scale = 1.5 / math.sqrt(float((g64 ** 2).sum(1).mean()))   # gates of about 1.5
    for dtype, left, right, pad, act in ((torch.float32, 4, 4, 0, "silu"),
                                         (torch.bfloat16, 8, 0, 8, "gelu"),
                                         (torch.bfloat16, 4, 8, 0, "silu")):
        wide = torch.full((m, k + pad), math.nan, dtype=torch.bfloat16, device=dev)
        x = wide[:, :k]
        x.copy_(_bf16(dev, gen, (m, k), scale))
        big = torch.full((m + 1, left + n + right), 7.0, dtype=dtype, device=dev)
        rt.gated_linear(x, gate, up, big[:m, left:left + n], activation=act)
        torch.cuda.synchronize()
        pj.check(big[:m, left:left + n], *pj.gated(pj.f64(x), g64, u64, act, dtype))
        assert (big[:m, :left] == 7.0).all() and (big[:m, left + n:] == 7.0).all()
        assert (big[m] == 7.0).all()


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_activations_over_their_range(dev, act):
    """Gates from -200 to 200 through one column, ups 1: the activation itself."""
    n, k = 1024, 64
    gate = torch.zeros((n, k), dtype=torch.bfloat16, device=dev)
    gate[:, 0] = torch.linspace(-200, 200, n, device=dev)
    gate[::2, 0] /= 16
    up = torch.zeros_like(gate)
    up[:, 1] = 1.0
    x = torch.zeros((1, k), dtype=torch.bfloat16, device=dev)
    x[0, :2] = 1.0
    out = torch.empty((1, n), dtype=torch.float32, device=dev)
    rt.gated_linear(x, gate, up, out, activation=act)
    g = pj.f64(gate[:, 0])
    want = of.activate(g, act)
    y = np.abs(g) if act == "silu" else np.abs(1.6 * (g + 0.044715 * g ** 3))
    bound = np.abs(want) * (4 * y + 10) * 2.0 ** -24 + 1e-36   # (e^-y past 2^126: 0 or subnormal)
    pj.check(out[0], want, bound)


@pytest.mark.parametrize("m", [1, 16, 40, 300])
@pytest.mark.parametrize("kind", ["linear4", "gated", "gated4"])
def test_values_that_are_not_finite_stay_in_their_rows_and_columns(dev, m, kind):
    """A token with an infinite or NaN value, and a feature with a NaN weight: only their outputs
    are not finite."""
    n, k = 96, 320
    gen = _gen(dev, m)
    x = _bf16(dev, gen, (m, k))
    token, feature = m // 2, 37
    out = torch.empty((m, n), dtype=torch.float32, device=dev)
    if kind == "gated":
        ws = [_bf16(dev, gen, (n, k), 0.05) for _ in range(2)]
        call = lambda: rt.gated_linear(x, *ws, out)  # noqa: E731
    else:
        ws = [_weights4(dev, gen, n, k) for _ in range(1 if kind == "linear4" else 2)]
        call = ((lambda: rt.linear(x, ws[0], out)) if kind == "linear4" else
                (lambda: rt.gated_linear(x, *ws, out)))
    call()
    clean = out.clone()
    x[token, k - 1] = math.nan
    if m > 2:
        x[token + 1, 0] = math.inf
    (ws[-1] if kind == "gated" else ws[-1].exps)[feature, 2] = math.nan if kind == "gated" else 255
    call()
    fine = torch.ones((m, n), dtype=torch.bool, device=dev)
    fine[token] = False
    if m > 2:
        fine[token + 1] = False
    fine[:, feature] = False
    assert torch.equal(out[fine], clean[fine])
    assert out[token].isnan().all() and out[:, feature].isnan().all()
    if m > 2:
        assert not out[token + 1].isfinite().any()


def test_calls_are_repeatable(dev):
    gen = _gen(dev, 5)
    for m, n, k in ((3, 512, 4096), (70, 1008, 1088), (600, 768, 512)):
        x = _bf16(dev, gen, (m, k))
        gate, up = _weights4(dev, gen, n, k), _weights4(dev, gen, n, k)
        outs = [torch.empty((m, n), dtype=torch.float32, device=dev) for _ in range(2)]
        for out in outs:
            rt.gated_linear(x, gate, up, out)
        assert torch.equal(*outs)


@pytest.mark.parametrize("m", [1, 48, 520])
@pytest.mark.parametrize("four", [False, True])
def test_feed_forward_block(dev, m, four):
    """Gate, up, activation, product, then down, the hidden rows left in bf16 between them; the
    weights to 4 bits on the way."""
    hidden, mlp = 512, 1344
    gen = _gen(dev, m)
    dense = [_bf16(dev, gen, s, 1.0 / math.sqrt(s[1])) for s in ((mlp, hidden), (mlp, hidden),
                                                                 (hidden, mlp))]
    ws = dense
    if four:
        ws = [rt.Weights4.from_bf16(w) for w in dense]
        for w, d in zip(ws, dense):
            w.dequantize(d)
    x = _bf16(dev, gen, (m, hidden))
    h = torch.empty((m, mlp), dtype=torch.bfloat16, device=dev)
    out = torch.empty((m, hidden), dtype=torch.float32, device=dev)
    rt.gated_linear(x, ws[0], ws[1], h)
    if four or hidden % 128 == 0:
        rt.linear(h, ws[2], out)
    torch.cuda.synchronize()
    pj.check(h, *pj.gated(pj.f64(x), pj.f64(dense[0]), pj.f64(dense[1]), "silu", torch.bfloat16))
    pj.check(out, *pj.linear(pj.f64(h), pj.f64(dense[2]), torch.float32))


def test_gate_and_up_halves_of_one_buffer(dev):
    gen = _gen(dev, 77)
    n, k, m = 208, 256, 37
    both = _bf16(dev, gen, (2 * n, k), 0.1)
    x = _bf16(dev, gen, (m, k))
    a, b, c = (torch.empty((m, n), dtype=torch.bfloat16, device=dev) for _ in range(3))
    rt.gated_linear(x, both[:n], both[n:], a)
    rt.gated_linear(x, both[:n].clone(), both[n:].clone(), b)
    rt.gated_linear(x, both[n:], both[:n], c)
    assert torch.equal(a, b)
    pj.check(c, *pj.gated(pj.f64(x), pj.f64(both[n:]), pj.f64(both[:n]), "silu", torch.bfloat16))


# ------------------------------------------------------------------- streams, graphs, far addresses

@pytest.mark.parametrize("m", [1, 24, 300])
def test_graph_replays(dev, m):
    """A captured block (quantised weights, gated, down) replayed with new inputs, eager work
    between the replays."""
    hidden, mlp = 256, 16384
    gen = _gen(dev, m + 100)
    ws = [rt.Weights4.from_bf16(_bf16(dev, gen, s, 0.06)) for s in ((mlp, hidden), (mlp, hidden),
                                                                    (hidden, mlp))]
    x = _bf16(dev, gen, (m, hidden))
    h = torch.empty((m, mlp), dtype=torch.bfloat16, device=dev)
    out, eager = (torch.empty((m, hidden), dtype=torch.float32, device=dev) for _ in range(2))
    if m > 1:
        assert D.dlfp_projection_workspace(D.LINEAR_W4, m, hidden, mlp) > 0

    def block(y):
        rt.gated_linear(x, ws[0], ws[1], h)
        rt.linear(h, ws[2], y)

    block(eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block(out)
    for _ in range(4):
        x.copy_(_bf16(dev, gen, (m, hidden)))
        graph.replay()
        torch.cuda.synchronize()
        kept = out.clone()
        block(eager)
        torch.cuda.synchronize()
        assert torch.equal(kept, eager)


def test_two_streams_at_once(dev):
    gen = _gen(dev, 9)
    n, k, m = 1024, 2048, 64
    w = [_weights4(dev, gen, n, k) for _ in range(2)]
    xs = [_bf16(dev, gen, (m, k)) for _ in range(2)]
    want = [torch.empty((m, n), dtype=torch.float32, device=dev) for _ in range(2)]
    got = [torch.empty_like(t) for t in want]
    for i in range(2):
        rt.linear(xs[i], w[i], want[i])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(8):
        for i, s in enumerate(streams):
            rt.linear(xs[i], w[i], got[i], stream=s)
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(got[i], want[i])


def test_two_current_streams_and_their_graphs(dev):
    """K over workgroups on two current streams at once, eager and as a graph of each replayed
    beside the other: every call has partial sums of its own."""
    gen = _gen(dev, 19)
    m, n, k = 256, 1024, 16384
    for kind in (D.LINEAR_W4, D.GATED_LINEAR_BF16, D.GATED_LINEAR_W4):
        assert D.dlfp_projection_workspace(kind, m, n, k) > 0
    w = [_weights4(dev, gen, n, k) for _ in range(2)]
    dense = [_bf16(dev, gen, (n, k), 0.02) for _ in range(2)]
    xs = [_bf16(dev, gen, (m, k)) for _ in range(2)]
    outs = [[torch.empty((m, n), dtype=torch.float32, device=dev) for _ in range(3)]
            for _ in range(2)]

    def block(i):
        rt.linear(xs[i], w[i], outs[i][0])
        rt.gated_linear(xs[i], dense[i], dense[1 - i], outs[i][1])
        rt.gated_linear(xs[i], w[i], w[1 - i], outs[i][2], "gelu")

    def take():
        torch.cuda.synchronize()
        kept = [[t.clone() for t in ts] for ts in outs]
        for ts in outs:
            for t in ts:
                t.fill_(math.nan)
        torch.cuda.synchronize()
        return kept

    for i in range(2):
        block(i)
    want = take()
    streams = [torch.cuda.Stream() for _ in range(2)]
    graphs = []
    for i, s in enumerate(streams):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i], stream=s):
            block(i)
    for eager in (True, False, True, False):
        for _ in range(3):
            for i, s in enumerate(streams):
                with torch.cuda.stream(s):
                    block(i) if eager else graphs[i].replay()
        for got, expected in zip(take(), want):
            for t, u in zip(got, expected):
                assert torch.equal(t, u)


def test_weights_past_four_gigabytes(dev):
    """Row offsets past 32 bits: the last rows of weights of over 2^32 bytes."""
    gen = _gen(dev, 21)
    k, rows = 16448, 48
    n = 131088                                   # 2 n k > 2^32
    gate = torch.zeros((n, k), dtype=torch.bfloat16, device=dev)
    up = torch.zeros_like(gate)
    gate[-rows:] = _bf16(dev, gen, (rows, k), 0.01)
    up[-rows:] = _bf16(dev, gen, (rows, k), 0.01)
    for m in (1, 150):
        x = _bf16(dev, gen, (m, k))
        out = torch.empty((m, n), dtype=torch.bfloat16, device=dev)
        rt.gated_linear(x, gate, up, out)
        pj.check(out[:, -rows:], *pj.gated(pj.f64(x), pj.f64(gate[-rows:]), pj.f64(up[-rows:]),
                                           "silu", torch.bfloat16))
        assert not out[:, :-rows].any()
    del gate, up
    n = 524352                                   # n k / 2 > 2^32
    codes = torch.zeros((n, k // 2), dtype=torch.uint8, device=dev)
    exps = torch.full((n, k // 32), 120, dtype=torch.uint8, device=dev)
    codes[-rows:], exps[-rows:] = pj.random_codes(gen, rows, k, device=dev)
    w = rt.Weights4.of(codes, exps)
    values = of.values(codes[-rows:].cpu().numpy(), exps[-rows:].cpu().numpy())
    for m in (1, 150):
        x = _bf16(dev, gen, (m, k))
        out = torch.empty((m, n), dtype=torch.bfloat16, device=dev)
        rt.linear(x, w, out)
        pj.check(out[:, -rows:], *pj.linear(pj.f64(x), values, torch.bfloat16))
        assert not out[:, :-rows].any()


@pytest.mark.parametrize("m", [5, 67, 400])
def test_far_rows(dev, m):
    """Rows of x and out 2^22 elements and more apart: offsets past 32 bits."""
    gen = _gen(dev, 3)
    n, k, ld = 256, 192, (1 << 22) + 8
    x = torch.empty(((m - 1) * ld + k,), dtype=torch.bfloat16, device=dev).as_strided((m, k), (ld, 1))
    x.copy_(_bf16(dev, gen, (m, k)))
    out = torch.empty(((m - 1) * ld + n,), dtype=torch.bfloat16, device=dev).as_strided((m, n),
                                                                                        (ld, 1))
    w = _weights4(dev, gen, n, k)
    rt.linear(x, w, out)
    pj.check(out, *pj.linear(pj.f64(x), _values(w), torch.bfloat16))
    gate, up = (_bf16(dev, gen, (n, k), 0.1) for _ in range(2))
    rt.gated_linear(x, gate, up, out)
    pj.check(out, *pj.gated(pj.f64(x), pj.f64(gate), pj.f64(up), "silu", torch.bfloat16))


@pytest.mark.parametrize("m", [1, 3, 90])
def test_far_rows_of_one_side(dev, m):
    """4-bit gate and up with far rows of x; far rows of out, x's beside each other; a single
    row of a far view."""
    gen = _gen(dev, 4)
    n, k, ld = 96, 320, (1 << 22) + 16
    far = lambda cols: torch.empty(((m - 1) * ld + cols,), dtype=torch.bfloat16,
                                   device=dev).as_strided((m, cols), (ld, 1))
    near, x = _bf16(dev, gen, (m, k)), far(k)
    x.copy_(near)
    gate, up, out, one = _weights4(dev, gen, n, k), _weights4(dev, gen, n, k), far(n), far(n)
    rt.gated_linear(x, gate, up, out, "gelu")
    want = pj.gated(pj.f64(x), _values(gate), _values(up), "gelu", torch.bfloat16)
    pj.check(out, *want)
    rt.gated_linear(near, gate, up, one, "gelu")
    pj.check(one, *want)
    rt.linear(near, gate, one)
    pj.check(one, *pj.linear(pj.f64(near), _values(gate), torch.bfloat16))
    rt.linear(x[m - 1:], gate, one[m - 1:])
    pj.check(one[m - 1:], *pj.linear(pj.f64(near[m - 1:]), _values(gate), torch.bfloat16))


def test_many_tokens(dev):
    """More tokens than a grid's second dimension has blocks of 16."""
    gen = _gen(dev, 31)
    m, n, k = 16 * 65536 + 3, 16, 64
    x = _bf16(dev, gen, (m, k))
    w = _weights4(dev, gen, n, k)
    out = torch.empty((m, n), dtype=torch.float32, device=dev)
    rt.linear(x, w, out)
    for rows in (slice(0, 64), slice(m - 64, m)):
        pj.check(out[rows], *pj.linear(pj.f64(x[rows]), _values(w), torch.float32))
    gate, up = (_bf16(dev, gen, (n, k), 0.1) for _ in range(2))
    rt.gated_linear(x, gate, up, out)
    for rows in (slice(0, 64), slice(m - 64, m)):
        pj.check(out[rows], *pj.gated(pj.f64(x[rows]), pj.f64(gate), pj.f64(up), "silu",
                                      torch.float32))
