"""Performance cases of 4-bit weights and of the gated feed-forward projections.

Each case is one step that a serving program makes for a layer's projections
(x is bf16 [m][k], a row for each token of the iteration; weights have a row
for each output feature):

- kind "linear4": out = x W^T with 4-bit weights (`dlfp_linear_w4`);
- kind "gated": out = act(x G^T) * (x U^T) with bf16 weights
  (`dlfp_gated_linear_bf16`);
- kind "gated4": the same with 4-bit weights (`dlfp_gated_linear_w4`);
- kind "quantize": a bf16 weight to 4 bits, and the values that the codes stand
  for back in bf16 (`dlfp_quantize_w4`, `dlfp_dequantize_w4`), as a program does
  when it loads a model.

A 4-bit weight is an e2m1 code (sign, values 0 0.5 1 1.5 2 3 4 6; two to a byte,
the even column in the low half) times 2^(byte - 127), with an exponent byte for
each 32 columns of a row.  Of a group the exponent is the least that leaves its
largest magnitude at 6 or below, and codes are the nearest ones, ties to even.

Activations are N(0, 1), weights N(0, 1 / k).  Sizes are those of the layers that
the chunk-size sweeps' models have (hidden 1024 / 4096 / 5120) or generic ones;
`pad` elements lie between the rows of x where it is a part of wider rows.
"""
import math

import torch

own = False

GROUP = 32
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EXP_MIN, EXP_MAX, EXP_BIAS = -125, 125, 127
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _linear4(m, n, k, out="bf16", pad=0):
    return {"kind": "linear4", "m": m, "n": n, "k": k, "out": out, "pad": pad}


def _gated(kind, m, n, k, act="silu", out="bf16", pad=0):
    return {"kind": kind, "m": m, "n": n, "k": k, "act": act, "out": out, "pad": pad}


def _quantize(n, k):
    return {"kind": "quantize", "n": n, "k": k}


def listed():
    return [
        # One token of a nearly idle server through a small model's query projection.
        {"name": "linear4-one", **_linear4(1, 2048, 1024)},
        # One token through an 8B model's down projection: the weights' bytes.
        {"name": "linear4-vector", **_linear4(1, 4096, 12288)},
        # A decode batch through a 32B model's down projection, summed on in fp32.
        {"name": "linear4-decode", **_linear4(32, 5120, 25600, out="fp32")},
        # A short chunk beside decoders, sizes off every tile, x a part of wider rows.
        {"name": "linear4-ragged", **_linear4(77, 1008, 4160, pad=72)},
        # A prompt chunk through an 8B model's down projection.
        {"name": "linear4-chunk", **_linear4(2048, 4096, 12288)},
        # One token through a small model's gate and up.
        {"name": "gated-one", **_gated("gated", 1, 2816, 1024)},
        # A full decode batch of an 8B model: 201 MB of weights.
        {"name": "gated-decode", **_gated("gated", 64, 12288, 4096)},
        # A large prompt chunk of an 8B model: matrix cores.
        {"name": "gated-chunk", **_gated("gated", 4096, 12288, 4096)},
        # Eight decoders of a 32B model.
        {"name": "gated4-decode", **_gated("gated4", 8, 25600, 5120)},
        # A capped chunk beside 33 decoders of an 8B model, the other activation.
        {"name": "gated4-mixed", **_gated("gated4", 545, 12288, 4096, act="gelu")},
        # A small projection to 4 bits.
        {"name": "quantize-small", **_quantize(1024, 2048)},
        # A 32B model's gate projection to 4 bits.
        {"name": "quantize-large", **_quantize(25600, 5120)},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["linear4", "linear4", "gated", "gated4", "gated4", "quantize"])
    n = 16 * _log_int(rng, 4, 1600)
    k = 64 * _log_int(rng, 1, 400)
    # No more weights than the largest listed ones.
    n = max(16, min(n, 25600 * 5120 // k // 16 * 16))
    if kind == "quantize":
        return _quantize(n, k)
    m = _log_int(rng, 1, 4096)
    # No more products than the largest listed ones.
    m = max(1, min(m, 4096 * 12288 * 4096 * (2 if kind == "linear4" else 1) // (n * k)))
    out = rng.choice(["bf16", "bf16", "fp32"])
    pad = rng.choice([0, 0, 8 * rng.randint(1, 40)])
    if kind == "linear4":
        return _linear4(m, n, k, out, pad)
    return _gated(kind, m, n, k, rng.choice(["silu", "silu", "gelu"]), out, pad)


# ----------------------------------------------------------------- inputs

def _device():
    return torch.device("cuda:0" if torch.cuda.is_available() else "cpu")


def _generator(seed, salt=0):
    return torch.Generator(device=_device()).manual_seed(1000003 * int(seed) + salt)


def _weight(case, seed, salt):
    n, k = case["n"], case["k"]
    w = torch.empty((n, k), dtype=torch.float32, device=_device())
    return w.normal_(generator=_generator(seed, salt)).mul_(1.0 / math.sqrt(k)).to(torch.bfloat16)


def _tokens(case, seed):
    m, k = case["m"], case["k"]
    wide = torch.empty((m, k + case["pad"]), dtype=torch.bfloat16, device=_device())
    return wide.normal_(generator=_generator(seed))[:, :k]


def _to_codes(w):
    """bf16 [n][k] -> (codes uint8 [n][k / 2], exponent bytes uint8 [n][k / 32])."""
    n, k = w.shape
    x = w.float().view(n, k // GROUP, GROUP)
    mantissa, power = torch.frexp(x.abs().amax(-1))   # amax = mantissa 2^power, mantissa >= 1/2
    exps = torch.where(mantissa <= 0.75, power - 3, power - 2)       # 6 = 0.75 * 2^3
    exps = torch.where(mantissa > 0, exps, EXP_MIN).clamp(EXP_MIN, EXP_MAX)
    x = torch.ldexp(x, -exps[..., None])
    size = x.abs()
    # Midpoints between neighbouring magnitudes; a tie goes to the even code.
    code = ((size > 0.25).int() + (size >= 0.75) + (size > 1.25) + (size >= 1.75) + (size > 2.5) +
            (size >= 3.5) + (size > 5.0))
    code += 8 * torch.signbit(x)
    code = code.to(torch.uint8).view(n, k // 2, 2)
    return code[..., 0] | code[..., 1] << 4, (exps + EXP_BIAS).to(torch.uint8)


def prepare(case, seed):
    s = {"case": case}
    n, k = case["n"], case["k"]
    if case["kind"] == "quantize":
        s["w"] = _weight(case, seed, 1)
        s["values"] = torch.empty((n, k), dtype=torch.bfloat16, device=_device())
        if own:
            from paper_2609_38386_amd import runtime
            s["runtime"] = runtime
            s["weights"] = runtime.Weights4(n, k, _device())
        return s
    s["x"] = _tokens(case, seed)
    s["out"] = torch.empty((case["m"], n), dtype=DTYPES[case["out"]], device=_device())
    weights = [_weight(case, seed, salt) for salt in ((1,) if case["kind"] == "linear4" else (1, 2))]
    if case["kind"] != "gated":
        weights = [_to_codes(w) for w in weights]
    if own:
        from paper_2609_38386_amd import runtime
        s["runtime"] = runtime
        if case["kind"] != "gated":
            weights = [runtime.Weights4.of(codes, exps) for codes, exps in weights]
    s["weights"] = weights
    return s


def run(s):
    case = s["case"]
    if case["kind"] == "quantize":
        if own:
            s["weights"].quantize(s["w"])
            s["weights"].dequantize(s["values"])
            return [s["values"], s["weights"].exps]
        codes, exps = _to_codes(s["w"])
        return [_values(codes, exps).to(torch.bfloat16), exps]
    if own:
        if case["kind"] == "linear4":
            s["runtime"].linear(s["x"], s["weights"][0], s["out"])
        else:
            s["runtime"].gated_linear(s["x"], *s["weights"], s["out"], activation=case["act"])
        return [s["out"]]
    x = s["x"].float()
    if case["kind"] == "linear4":
        y = x @ _values(*s["weights"][0]).T
    else:
        gate, up = (w.float() if case["kind"] == "gated" else _values(*w) for w in s["weights"])
        y = _activate(x @ gate.T, case["act"]) * (x @ up.T)
    return [y.to(DTYPES[case["out"]])]


# ----------------------------------------------------------------- plain forms

def _values(codes, exps):
    """What 4-bit weights stand for, fp32 [n][k]."""
    table = torch.tensor(MAGNITUDES + tuple(-x for x in MAGNITUDES), device=codes.device)
    code = torch.stack([codes & 15, codes >> 4], -1).int()
    value = table[code].view(exps.shape[0], -1, GROUP)
    return torch.ldexp(value, exps.int()[..., None] - EXP_BIAS).flatten(1)


def _activate(g, act):
    if act == "silu":
        return g / (1.0 + torch.exp(-g))
    t = math.sqrt(2.0 / math.pi) * (g + 0.044715 * g * g * g)
    return g / (1.0 + torch.exp(-2.0 * t))


# ----------------------------------------------------------------- work and exact results

def work(case):
    n, k = case["n"], case["k"]
    four_bits = n * k // 2 + n * k // GROUP
    if case["kind"] == "quantize":      # to 4 bits and back
        return {"bytes": 2 * (2 * n * k + four_bits), "flops": 4 * n * k}
    m, products = case["m"], 1 if case["kind"] == "linear4" else 2
    weights = products * (2 * n * k if case["kind"] == "gated" else four_bits)
    rows = m * (2 * k + n * (4 if case["out"] == "fp32" else 2))
    return {"bytes": weights + rows, "flops": 2 * products * m * n * k}


def _exact_values(codes, exps):
    """The value of each code from its fields: 2 exponent bits of bias 1, a mantissa bit."""
    code = torch.stack([codes & 15, codes >> 4], -1).view(*exps.shape, GROUP).double()
    sign = torch.where(code >= 8, -1.0, 1.0)
    field = code % 8
    power, half = torch.floor(field / 2), field % 2
    size = torch.where(power > 0, (1.0 + half / 2) * torch.exp2(power - 1), half / 2)
    return (sign * size * torch.exp2(exps.double() - EXP_BIAS)[..., None]).flatten(1)


def _exact_nearest(w):
    """Each value's nearest 4-bit value, 64 bits."""
    x = w.double().view(w.shape[0], -1, GROUP)
    most = x.abs().amax(-1, keepdim=True)
    power = torch.ceil(torch.log2(most / 6.0)).clamp(EXP_MIN, EXP_MAX)
    power = torch.where(most > 0, power, float(EXP_MIN))
    x = x * torch.exp2(-power)
    # Steps of 1/2 below 2, of 1 below 4, of 2 up to 6.
    step = torch.where(x.abs() < 2, 0.5, torch.where(x.abs() < 4, 1.0, 2.0))
    return ((torch.round(x / step) * step).clamp(-6, 6) * torch.exp2(power)).flatten(1)


def exact(case, seed):
    if case["kind"] == "quantize":
        return [_exact_nearest(_weight(case, seed, 1)), None]
    x = _tokens(case, seed).double()

    def product(salt):
        w = _weight(case, seed, salt)
        w = w.double() if case["kind"] == "gated" else _exact_values(*_to_codes(w))
        return torch.matmul(x, w.t())

    y = product(1)
    if case["kind"] != "linear4":
        if case["act"] == "silu":
            y = y * torch.sigmoid(y)
        else:
            y = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y ** 3)))
        y = y * product(2)
    return [y]
