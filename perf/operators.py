"""Measured cases of the block-scaled operators: a layer's activations and weights on their way into low-precision products.

Three operators that follow one another in a program that serves a language model with 4-bit weights: the root-mean-square
norm with the residual's addition, whose output leaves in 8 bits with E8M0 scales (kind "norm"); weights brought to FP4
with group scales, MXFP4 or NVFP4 (kind "quantize"); and the product of activations with such weights, from one token to
a whole prompt (kind "product").  Each case is one call of one operator on one layer's data.

`run` computes the plain form in elementary torch operations where `own` is false, and makes the library's calls where it
is true.  8-bit codes and scale codes are returned as the float8 types whose bytes they are; packed FP4 codes as the
numbers that they and their scales stand for (the operator writes those too, for programs that evaluate a quantised model).
"""
import math

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4, "e4m3": 1, "e5m2": 1}
BLOCK = {"e8m0": 32, "ue4m3": 16}                   # elements of a row that share a scale
EPS = 1e-6
STD = 0.02                                          # of the weights
# NVFP4's scale per tensor, a binary32 number: a weight of six standard deviations comes to 6 x 448
TENSOR_SCALE = torch.tensor(6 * STD / (6 * 448), dtype=torch.float32).item()


def listed():
    return [
        # One token between two layers of a served model: latency.
        dict(name="norm_token_bf16", kind="norm", type="bf16", code="e4m3", rule="floor", rows=1, cols=4096, pad=0, residual=True),
        # A decoding batch, FP16 activations, E5M2 codes, scales that never saturate.
        dict(name="norm_batch_fp16", kind="norm", type="fp16", code="e5m2", rule="fit", rows=96, cols=8192, pad=0, residual=True),
        # A prompt of 8192 tokens: bound by memory.
        dict(name="norm_prompt_bf16", kind="norm", type="bf16", code="e4m3", rule="floor", rows=8192, cols=8192, pad=0, residual=True),
        # Binary32 activations, rows of an odd length that are slices of wider ones, no residual stream.
        dict(name="norm_ragged_fp32", kind="norm", type="fp32", code="e4m3", rule="fit", rows=1537, cols=2731, pad=5, residual=False),
        # One projection's weights to MXFP4, with the values they then stand for.
        dict(name="quantize_mx_bf16", kind="quantize", type="bf16", scale="e8m0", rule="fit", rows=4096, cols=4096, pad=0),
        # Binary32 master weights to NVFP4 with a scale per tensor; rows that end inside a group.
        dict(name="quantize_nv_ragged", kind="quantize", type="fp32", scale="ue4m3", rule="floor", rows=11003, cols=5000, pad=0),
        # One token through one projection, weights only in 4 bits: the smallest product.
        dict(name="token_bf16_mx", kind="product", a="bf16", d="bf16", scale="e8m0", m=1, n=4096, k=4096, pad=0),
        # One token in 8 bits through a wide layer: the stream of the weights is all there is.
        dict(name="token_fp8_mx", kind="product", a="e4m3", d="bf16", scale="e8m0", m=1, n=28672, k=8192, pad=0),
        # A decoding batch on NVFP4 weights; the activations are a slice of a wider buffer.
        dict(name="batch_fp16_nv", kind="product", a="fp16", d="fp16", scale="ue4m3", m=16, n=8192, k=8192, pad=64),
        # A ragged batch with a binary32 result: no dimension a multiple of a tile.
        dict(name="ragged_bf16_mx", kind="product", a="bf16", d="fp32", scale="e8m0", m=77, n=5003, k=4128, pad=0),
        # Prompts: 2048 tokens with 16-bit activations, 8192 in 8 bits.
        dict(name="prompt_bf16_mx", kind="product", a="bf16", d="bf16", scale="e8m0", m=2048, n=8192, k=4096, pad=0),
        dict(name="prompt_fp8_mx", kind="product", a="e4m3", d="bf16", scale="e8m0", m=8192, n=8192, k=8192, pad=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("norm", "quantize", "product", "product"))
    while True:
        if kind == "norm":
            c = dict(kind=kind, type=rng.choice(("bf16", "bf16", "fp16", "fp32")), code=rng.choice(("e4m3", "e4m3", "e5m2")), rule=rng.choice(("floor", "fit")),
                     rows=_log(rng, 1, 8192), cols=_log(rng, 100, 16384), pad=rng.choice((0, 0, 8, 3)), residual=rng.random() < 0.7)
            if rng.random() < 0.6:
                c["cols"] = max(128, c["cols"] // 128 * 128)
            if c["rows"] * c["cols"] <= 1 << 25:
                return c
        elif kind == "quantize":
            c = dict(kind=kind, type=rng.choice(("bf16", "bf16", "fp16", "fp32")), scale=rng.choice(("e8m0", "ue4m3")), rule="floor",
                     rows=_log(rng, 64, 32768), cols=_log(rng, 64, 16384), pad=rng.choice((0, 0, 8, 3)))
            if c["scale"] == "e8m0":
                c["rule"] = rng.choice(("floor", "fit"))
            if rng.random() < 0.6:
                c["cols"] = max(64, c["cols"] // 64 * 64)
            if c["rows"] * c["cols"] <= 1 << 26:
                return c
        else:
            a = rng.choice(("bf16", "bf16", "fp16", "e4m3", "e4m3", "e5m2"))
            c = dict(kind=kind, a=a, d=rng.choice(("bf16", "fp16", "fp32") if SIZE[a] == 2 else ("bf16", "fp16")),
                     scale=rng.choice(("e8m0", "e8m0", "ue4m3")) if SIZE[a] == 2 else "e8m0",
                     m=_log(rng, 1, 8192), n=_log(rng, 200, 32768), k=32 * _log(rng, 8, 512), pad=rng.choice((0, 0, 64)))
            if rng.random() < 0.6:
                c["n"] = max(256, c["n"] // 64 * 64)
            if c["n"] * c["k"] <= 28672 * 8192 and c["m"] * c["n"] * c["k"] <= (1 << 39 if SIZE[a] == 1 else 1 << 37):
                return c


def work(case):
    if case["kind"] == "norm":
        e, cols = case["rows"] * case["cols"], case["cols"]
        t = SIZE[case["type"]]
        return {"bytes": e * (t * (3 if case["residual"] else 1) + 1) + case["rows"] * -(-cols // 32) + cols * t, "flops": 6 * e}
    if case["kind"] == "quantize":
        e, t = case["rows"] * case["cols"], SIZE[case["type"]]
        return {"bytes": e * 2 * t + e // 2 + case["rows"] * -(-case["cols"] // BLOCK[case["scale"]]), "flops": 4 * e}
    m, n, k = case["m"], case["n"], case["k"]
    a = m * k * SIZE[case["a"]] + (m * k // 32 if SIZE[case["a"]] == 1 else 0)
    return {"bytes": a + n * k // 2 + n * k // BLOCK[case["scale"]] + m * n * SIZE[case["d"]], "flops": 2 * m * n * k}


# ---- inputs -------------------------------------------------------------------------------

def _normal(shape, gen, dtype, std=1.0):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * std).to(dtype)


def _activations(rows, cols, gen, dtype):
    """Rows of different sizes, and a few channels that are far larger than the rest, as the residual stream has them."""
    x = torch.randn((rows, cols), generator=gen, device="cuda", dtype=torch.float32)
    x *= torch.exp(0.5 * torch.randn((rows, 1), generator=gen, device="cuda"))
    x[:, ::97] *= 8.0
    return x.to(dtype)


def _in_chunks(fn, x, rows=4096):
    """fn on blocks of rows, its tuple of results joined: the temporaries stay small."""
    parts = [fn(x[i:i + rows]) for i in range(0, x.shape[0], rows)]
    return [torch.cat(p) for p in zip(*parts)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case=case)
    if case["kind"] == "norm":
        rows, cols, t = case["rows"], case["cols"], TYPES[case["type"]]
        padded = -(-cols // 32) * 32
        s["x"] = _activations(rows, cols + case["pad"], gen, t)[:, :cols]
        s["residual"] = _activations(rows, cols + case["pad"], gen, t)[:, :cols] if case["residual"] else None
        s["weight"] = (1 + 0.2 * torch.randn(cols, generator=gen, device="cuda")).to(t)
        s["residual_out"] = torch.empty_strided((rows, cols), (cols + case["pad"], 1), dtype=t, device="cuda") if case["residual"] else None
        s["codes"] = torch.empty((rows, padded), dtype=torch.uint8, device="cuda")
        s["scales"] = torch.empty((rows, padded // 32), dtype=torch.uint8, device="cuda")
    elif case["kind"] == "quantize":
        rows, cols, t, b = case["rows"], case["cols"], TYPES[case["type"]], BLOCK[case["scale"]]
        padded = -(-cols // 32) * 32
        s["x"] = _normal((rows, cols + case["pad"]), gen, t, STD)[:, :cols]
        s["tensor_scale"] = TENSOR_SCALE if case["scale"] == "ue4m3" else 1.0
        s["codes"] = torch.empty((rows, padded // 2), dtype=torch.uint8, device="cuda")
        s["scales"] = torch.empty((rows, padded // b), dtype=torch.uint8, device="cuda")
        s["values"] = torch.empty((rows, cols), dtype=t, device="cuda")
    else:
        m, n, k, pad = case["m"], case["n"], case["k"], case["pad"]
        s["alpha"] = TENSOR_SCALE if case["scale"] == "ue4m3" else 1.0
        w = _normal((n, k), gen, torch.bfloat16, STD)
        s["W"], s["SW"] = _in_chunks(lambda x: _quantize_plain(x, case["scale"], "fit", s["alpha"])[:2], w)
        if SIZE[case["a"]] == 2:
            s["A"], s["SA"] = _activations(m, k + pad, gen, TYPES[case["a"]])[:, :k], None
        else:
            a, s["SA"] = _in_chunks(lambda x: _quantize8_plain(x.float(), case["a"], "floor"), _activations(m, k, gen, torch.bfloat16))
            wide = torch.zeros((m, k + pad), dtype=torch.uint8, device="cuda")
            wide[:, :k] = a
            s["A"] = wide[:, :k]
        s["D"] = torch.empty((m, n), dtype=TYPES[case["d"]], device="cuda")
    return s


# ---- the operators, plain -----------------------------------------------------------------

def _exponent(amax, rule, top, emax):
    """Exponent of a block's E8M0 scale: of the element type's largest power of two at the block's (floor), or the least with
    which nothing saturates (fit).  `top`: the largest element over 2^(emax + 1)."""
    mant, e = torch.frexp(amax)
    e = e - 1 - emax
    if rule == "fit":
        e = e + (mant > top).to(e.dtype)
    return torch.where(amax == 0, -127, e).clamp(-127, 127)


def _quantize8_plain(y, code, rule):
    """y (binary32, rows of a multiple of 32): codes and E8M0 codes, as bytes."""
    rows, cols = y.shape
    t = TYPES[code]
    top, emax = (448.0, 8) if code == "e4m3" else (57344.0, 15)
    v = y.reshape(rows, cols // 32, 32)
    e = _exponent(v.abs().amax(-1, keepdim=True), rule, top / 2.0 ** (emax + 1), emax)
    q = (v.double() * torch.exp2(-e.double())).clamp(-top, top).float().to(t)
    return q.view(torch.uint8).reshape(rows, cols), (e + 127).to(torch.uint8).reshape(rows, cols // 32)


def _norm_plain(s):
    case = s["case"]
    cols, t = case["cols"], TYPES[case["type"]]
    h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(t)
    d = h.double()
    # 64 bits: a value next to a border between two codes must not cross it
    y = (d * (1.0 / torch.sqrt((d * d).mean(-1, keepdim=True) + EPS)) * s["weight"].double()).float()
    y = torch.cat((y, y.new_zeros((y.shape[0], -cols % 32))), dim=1)
    codes, scales = _quantize8_plain(y, case["code"], case["rule"])
    out = dict(codes=codes.view(TYPES[case["code"]]), scales=scales.view(torch.float8_e8m0fnu))
    if s["residual"] is not None:
        out["residual"] = h
    return out


def _quantize_plain(x, scale, rule, tensor_scale):
    """Packed E2M1 codes, scale codes (bytes), and the values both stand for in binary64; rows padded to a multiple of 32."""
    rows, cols = x.shape
    b = BLOCK[scale]
    v = torch.cat((x.float(), x.new_zeros((rows, -cols % 32), dtype=torch.float32)), dim=1).reshape(rows, -1, b)
    amax = v.abs().amax(-1, keepdim=True)
    if scale == "e8m0":
        e = _exponent(amax, rule, 6.0 / 8.0, 2)
        scales, unit = (e + 127).to(torch.uint8), torch.exp2(e.double())
    else:
        # 64 bits: quotients next to a border between two codes.  E4M3 has units of 2^(exponent - 3), at least 2^-9; a sum
        # with 1.5 x 2^52 units is rounded at that place
        p = (amax.double() / (6.0 * tensor_scale)).clamp(max=448.0)
        far = torch.exp2(((torch.frexp(p)[1] - 4).clamp(min=-9) + 52).double()) * 1.5
        scales = ((p + far) - far).float().to(torch.float8_e4m3fn)
        unit = scales.double() * tensor_scale
        scales = scales.view(torch.uint8)
    q = torch.where(unit > 0, v.double() / unit, 0.0 * v.double())
    a = q.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)).to(torch.uint8)
    value = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device=x.device)[code.long()] * unit
    value = torch.where(torch.signbit(q), -value, value).reshape(rows, -1)[:, :cols]
    code = (code | (torch.signbit(q).to(torch.uint8) << 3)).reshape(rows, -1)
    return code[:, 0::2] | (code[:, 1::2] << 4), scales.reshape(rows, -1), value


def _product_plain(s):
    case = s["case"]
    n, k, b = case["n"], case["k"], BLOCK[case["scale"]]
    lut = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
    lut = torch.cat((lut, -lut))
    w = lut[torch.stack((s["W"] & 15, s["W"] >> 4), dim=-1).reshape(n, k).int()]
    sw = s["SW"].view(torch.float8_e8m0fnu if case["scale"] == "e8m0" else torch.float8_e4m3fn).float()
    w = (w.reshape(n, k // b, b) * sw.unsqueeze(-1)).reshape(n, k)
    if s["SA"] is None:
        a = s["A"].float()
    else:
        a = s["A"].contiguous().view(TYPES[case["a"]]).float().reshape(-1, k // 32, 32)
        a = (a * s["SA"].view(torch.float8_e8m0fnu).float().unsqueeze(-1)).reshape(-1, k)
    return (torch.mm(a, w.t()) * s["alpha"]).to(TYPES[case["d"]])


def run(s):
    case = s["case"]
    kind = case["kind"]
    if not own:
        if kind == "norm":
            return _norm_plain(s)
        if kind == "quantize":
            _, scales, value = _quantize_plain(s["x"], case["scale"], case["rule"], s["tensor_scale"])
            return dict(scales=scales.view(torch.float8_e8m0fnu if case["scale"] == "e8m0" else torch.float8_e4m3fn), values=value.to(s["x"].dtype))
        return _product_plain(s)
    from paper_2511_10909_amd import binding as mm
    ids = {"bf16": mm.BF16, "fp16": mm.FP16, "fp32": mm.FP32, "e4m3": mm.E4M3, "e5m2": mm.E5M2}
    rule = mm.SCALE_RULE_FIT if case.get("rule") == "fit" else mm.SCALE_RULE_FLOOR
    if kind == "norm":
        t, stride = ids[case["type"]], case["cols"] + case["pad"]
        mm.rmsnorm_quantize(s["x"], s["residual"], s["weight"], s["residual_out"], s["codes"], s["scales"], case["rows"], case["cols"], t, t,
                            ids[case["code"]], rule, EPS, stride, stride)
        out = dict(codes=s["codes"].view(TYPES[case["code"]]), scales=s["scales"].view(torch.float8_e8m0fnu))
        if s["residual"] is not None:
            out["residual"] = s["residual_out"]
        return out
    fmt = mm.SCALE_FORMAT_E8M0 if case["scale"] == "e8m0" else mm.SCALE_FORMAT_UE4M3
    if kind == "quantize":
        mm.quantize_fp4(s["x"], s["codes"], s["scales"], s["values"], case["rows"], case["cols"], ids[case["type"]], fmt, rule, s["tensor_scale"],
                        case["cols"] + case["pad"])
        return dict(scales=s["scales"].view(torch.float8_e8m0fnu if case["scale"] == "e8m0" else torch.float8_e4m3fn), values=s["values"])
    mm.matmul_fp4(s["A"], s["SA"], s["W"], s["SW"], s["D"], case["m"], case["n"], case["k"], ids[case["a"]], ids[case["d"]], fmt, s["alpha"],
                  case["k"] + case["pad"])
    return s["D"]


# ---- the same from the definitions, in 64 bits ----------------------------------------------

def _grid(v, mant, emin, top):
    """v rounded to the nearest multiple of its unit in the last place (ties to even), saturated: `mant` mantissa bits, least exponent `emin`."""
    _, e = torch.frexp(v)
    unit = torch.ldexp(torch.ones_like(v), torch.clamp(e - 1, min=emin) - mant)
    return torch.clamp(torch.round(v / unit) * unit, -top, top)


def _power_scale(amax, rule, top):
    """The power of two that a block with this largest magnitude is divided by."""
    _, et = torch.frexp(torch.tensor(top, dtype=torch.float64))
    _, e = torch.frexp(amax)
    p = torch.ldexp(torch.ones_like(amax), e - et)
    if rule == "fit":
        p = torch.where(amax > top * p, 2 * p, p)
    return torch.where(amax > 0, p, torch.full_like(p, 2.0 ** -127)).clamp(2.0 ** -127, 2.0 ** 127)


def _exact_norm(s):
    case = s["case"]
    rows, cols = case["rows"], case["cols"]
    h = s["x"].double()
    if s["residual"] is not None:
        h = (h + s["residual"].double()).to(TYPES[case["type"]]).double()     # the residual stream is held in its type
    y = torch.zeros((rows, -(-cols // 32) * 32), dtype=torch.float64, device=h.device)
    y[:, :cols] = h * s["weight"].double() / torch.sqrt(h.square().sum(1, keepdim=True) / cols + EPS)
    y = y.view(rows, -1, 32)
    mant, emin, top = (3, -6, 448.0) if case["code"] == "e4m3" else (2, -14, 57344.0)
    p = _power_scale(y.abs().max(dim=2, keepdim=True).values, case["rule"], top)
    out = dict(codes=_grid(y / p, mant, emin, top).view(rows, -1), scales=p.view(rows, -1))
    if s["residual"] is not None:
        out["residual"] = h
    return out


def _exact_quantize(s):
    case = s["case"]
    rows, cols, b = case["rows"], case["cols"], BLOCK[case["scale"]]
    v = torch.zeros((rows, -(-cols // 32) * 32), dtype=torch.float64, device=s["x"].device)
    v[:, :cols] = s["x"].double()
    v = v.view(rows, -1, b)
    amax = v.abs().max(dim=2, keepdim=True).values
    ts = s["tensor_scale"]
    p = _power_scale(amax, case["rule"], 6.0) if case["scale"] == "e8m0" else _grid(amax / 6.0 / ts, 3, -6, 448.0)
    q = _grid(v / torch.where(p > 0, p * ts, torch.full_like(p, math.inf)), 1, 0, 6.0)
    return dict(scales=p.view(rows, -1), values=(q * (p * ts)).view(rows, -1)[:, :cols])


def _bits(b, ebits, mbits, bias):
    """Bytes as the numbers they stand for (finite ones), sign on top of ebits + mbits bits."""
    b = b.int()
    e, m = (b >> mbits) & ((1 << ebits) - 1), b & ((1 << mbits) - 1)
    v = torch.ldexp((m + torch.where(e > 0, 1 << mbits, 0)).double(), e.clamp(min=1) - bias - mbits)
    return torch.where((b >> (ebits + mbits)) & 1 == 1, -v, v)


def _exact_product(s):
    case = s["case"]
    n, k, b = case["n"], case["k"], BLOCK[case["scale"]]
    w = torch.empty((n, k), dtype=torch.float64, device=s["W"].device)
    w[:, 0::2], w[:, 1::2] = _bits(s["W"] & 15, 2, 1, 1), _bits(s["W"] >> 4, 2, 1, 1)
    sw = torch.exp2(s["SW"].double() - 127) if case["scale"] == "e8m0" else _bits(s["SW"], 4, 3, 7)
    w *= sw.repeat_interleave(b, dim=1)
    if s["SA"] is None:
        a = s["A"].double()
    else:
        a = _bits(s["A"], *((4, 3, 7) if case["a"] == "e4m3" else (5, 2, 15))) * torch.exp2(s["SA"].double() - 127).repeat_interleave(32, dim=1)
    return torch.matmul(a, w.transpose(0, 1)) * s["alpha"]


def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "quantize": _exact_quantize, "product": _exact_product}[case["kind"]](s)
