"""Block-scaled operators in binary64 (numpy), from their definitions: RMS norm to 8-bit codes with E8M0 scales, weights to FP4
with E8M0 or UE4M3 group scales, and products of such operands.  Shares no code with the GPU path."""
import numpy as np

E4M3, E5M2, FP16, BF16, FP32 = 0, 1, 2, 3, 4
FLOOR, FIT = 0, 1
SCALE_E8M0, SCALE_UE4M3 = 0, 1
GRID = {E4M3: (3, -6, 448.0), E5M2: (2, -14, 57344.0), "E2M1": (1, 0, 6.0)}        # mantissa bits, least exponent, largest number


def bits_of(x, t):
    """Bit patterns (uint16 / uint32) of binary32 values rounded to type t, nearest even."""
    x = np.asarray(x, dtype=np.float32)
    if t == FP32:
        return x.view(np.uint32)
    if t == FP16:
        with np.errstate(over="ignore"):
            return x.astype(np.float16).view(np.uint16)
    b = x.view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FC0), r).astype(np.uint16)


def values_of(b, t):
    """Binary64 values of bit patterns of type t (FP32, FP16, BF16, E4M3, E5M2)."""
    b = np.asarray(b)
    if t == FP32:
        return b.view(np.float32).astype(np.float64)
    if t == FP16:
        return b.view(np.float16).astype(np.float64)
    if t == BF16:
        return (b.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    mb, emin, _ = GRID[t]
    e, m = (b.astype(np.int64) & 0x7F) >> mb, b.astype(np.int64) & ((1 << mb) - 1)
    v = np.ldexp((m + np.where(e > 0, 1 << mb, 0)).astype(np.float64), (np.maximum(e, 1) + emin - 1 - mb).astype(np.int32))
    if t == E4M3:
        v = np.where((b & 0x7F) == 0x7F, np.nan, v)
    else:
        v = np.where((b & 0x7F) == 0x7C, np.inf, np.where((b & 0x7F) > 0x7C, np.nan, v))
    return np.where(b & 0x80, -v, v)


def _codes(v, t):
    """Codes (sign on top) of finite binary64 values, nearest even, saturated."""
    mb, emin, top = GRID[t]
    a = np.minimum(np.abs(v), top)
    e = np.where(a > 0, np.maximum(np.frexp(a)[1] - 1, emin), emin)
    n = np.rint(np.ldexp(a, (mb - e).astype(np.int32))).astype(np.int64)         # multiples of the unit in the last place
    code = n + ((e - emin) << mb)                                                # a carry moves on into the exponent field
    width = {E4M3: 7, E5M2: 7, "E2M1": 3}[t]
    return (code | (np.signbit(v).astype(np.int64) << width)).astype(np.uint8)


def e8m0_codes(amax, t, rule):
    """Scale codes for blocks of largest magnitude amax (finite binary64)."""
    _, _, top = GRID[t]
    e = np.frexp(amax)[1] - np.frexp(top)[1]
    if rule == FIT:
        e = e + (amax > top * np.exp2(e.astype(np.float64)))
    return np.where(amax > 0, np.clip(e + 127, 0, 254), 0).astype(np.uint8)


def pad32(a):
    return np.concatenate([a, np.zeros((a.shape[0], -a.shape[1] % 32), dtype=a.dtype)], axis=1)


def quantize8(y, t, rule):
    """Binary32 values (rows of any length): (codes, scale codes), rows padded to multiples of 32."""
    y = pad32(np.asarray(y, dtype=np.float32).astype(np.float64))
    v = y.reshape(y.shape[0], -1, 32)
    bad = ~np.isfinite(v).all(-1)
    v = np.where(bad[..., None], 0.0, v)
    s = e8m0_codes(np.abs(v).max(-1), t, rule)
    q = _codes(np.ldexp(v, (127 - s.astype(np.int32))[..., None]), t)
    q = np.where(bad[..., None], np.uint8(0), q)
    return q.reshape(y.shape), np.where(bad, np.uint8(0xFF), s)


def rmsnorm(x, residual, weight, t, eps):
    """Bit patterns in (weight: values or None): (h as bit patterns, y as binary32)."""
    with np.errstate(all="ignore"):
        h = x if residual is None else bits_of(values_of(x, t).astype(np.float32) + values_of(residual, t).astype(np.float32), t)
        d = values_of(h, t)
        y = d * (1.0 / np.sqrt(np.mean(d * d, axis=1, keepdims=True) + eps))
        if weight is not None:
            y = y * np.asarray(weight, dtype=np.float64)
        return h, y.astype(np.float32)


def quantize_fp4(x, scale_format, rule, tensor_scale):
    """Finite or not, binary64 values: (packed codes, scale codes, values in binary64 without the padding)."""
    rows, cols = x.shape
    b = 32 if scale_format == SCALE_E8M0 else 16
    v = pad32(np.asarray(x, dtype=np.float64)).reshape(rows, -1, b)
    bad = ~np.isfinite(v).all(-1)
    v = np.where(bad[..., None], 0.0, v)
    amax = np.abs(v).max(-1)
    if scale_format == SCALE_E8M0:
        s = e8m0_codes(amax, "E2M1", rule)
        unit = np.exp2(s.astype(np.float64) - 127)
    else:
        s = _codes(amax / (6.0 * tensor_scale), E4M3)
        unit = values_of(s, E4M3) * tensor_scale
    with np.errstate(all="ignore"):
        q = np.where(unit[..., None] > 0, v / unit[..., None], np.copysign(0.0, v))
    c = np.where(bad[..., None], np.uint8(0), _codes(q, "E2M1"))
    val = np.where(bad[..., None], np.nan, fp4_values(c) * unit[..., None]).reshape(rows, -1)[:, :cols]
    c = c.reshape(rows, -1)
    return c[:, 0::2] | (c[:, 1::2] << 4), np.where(bad, np.uint8(0xFF if scale_format == SCALE_E8M0 else 0x7F), s), val


def fp4_values(c):
    return np.array([0, .5, 1, 1.5, 2, 3, 4, 6, -0.0, -.5, -1, -1.5, -2, -3, -4, -6])[c]


def unpack(w):
    return np.stack([w & 15, w >> 4], -1).reshape(w.shape[0], -1)


def scale_values(s, scale_format):
    if scale_format == SCALE_E8M0:
        return np.where(s == 0xFF, np.nan, np.exp2(s.astype(np.float64) - 127))
    return values_of(s & 0x7F, E4M3)


def weights(w, sw, scale_format):
    """Binary64 weights of packed codes and scale codes."""
    return fp4_values(unpack(w)) * np.repeat(scale_values(sw, scale_format), 32 if scale_format == SCALE_E8M0 else 16, axis=1)
