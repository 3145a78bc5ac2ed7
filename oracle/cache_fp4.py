"""The cache in 4 bits and its operators in binary64 (numpy), from their definitions: the pages' bytes, heads normed, rotated and appended, and
attention over what the cache holds.  Shares no code with the GPU path."""
import numpy as np

from . import block_scale as bs

HALVES, PAIRS = 0, 1
LEAST, MOST, NAN = 104, 140, 255


def places(d):
    """Byte of a granule for token t (32) and element pair (d / 2) of K and V codes, and for token t and block (d / 32) of their scales."""
    t, p, b = np.arange(32)[:, None], np.arange(0, d, 2)[None, :], np.arange(d // 32)[None, :]
    w, a, r = t // 8, t // 4 % 2, t % 4
    if d == 128:
        k = a * 1024 + p // 32 * 256 + (4 * w + r) * 16 + p % 32 // 2
        v = p // 4 % 2 * 1024 + w * 256 + p // 8 * 16 + p // 2 % 2 * 8 + t % 8
    else:
        k = p // 16 * 256 + (4 * w + r) * 16 + a * 8 + p % 16 // 2
        v = w * 256 + p // 4 * 16 + p // 2 % 2 * 8 + t % 8
    return k, 16 * d + v, 32 * d + (16 * b + 4 * w + r) * 2 + a, 33 * d + (w * (d // 32) + b) * 8 + t % 8


def quantize(y, rule):
    """Values [..., d] to codes (one a byte), scale codes, and the values that they stand for."""
    v = np.asarray(y, dtype=np.float64)
    v = v.reshape(v.shape[:-1] + (v.shape[-1] // 32, 32))
    bad = ~np.isfinite(v).all(-1)
    v = np.where(bad[..., None], 0.0, v)
    s = np.clip(bs.e8m0_codes(np.abs(v).max(-1), "E2M1", rule), LEAST, MOST)
    c = bs._codes(np.ldexp(v, (127 - s.astype(np.int32))[..., None]), "E2M1")
    c = np.where(bad[..., None], np.uint8(0), c)
    s = np.where(bad, np.uint8(NAN), s).astype(np.uint8)
    return c.reshape(np.shape(y)), s, values(c.reshape(np.shape(y)), s)


def values(codes, scales):
    return bs.fp4_values(codes) * np.repeat(bs.scale_values(scales, bs.SCALE_E8M0), 32, axis=-1)


def write(memory, table, page_tokens, t, k, ks, v, vs):
    """Token t of a sequence with pages `table`: its heads' codes k, v [kv][d] and scales into memory [pages][kv][granules][34 d]; no page, no writing."""
    page = int(table[t // page_tokens])
    if not 0 <= page < memory.shape[0]:
        return
    d = k.shape[-1]
    pk, pv, pks, pvs = (x[t % 32] for x in places(d))
    g = memory[page, :, t % page_tokens // 32]
    g[:, pk], g[:, pv] = k[:, 0::2] | (k[:, 1::2] << 4), v[:, 0::2] | (v[:, 1::2] << 4)
    g[:, pks], g[:, pvs] = ks, vs


def read(memory, table, page_tokens, length, d):
    """Keys and values [length][kv][d] in binary64, and which tokens have a page."""
    pages, kv = memory.shape[:2]
    pk, pv, pks, pvs = places(d)
    per = page_tokens // 32
    out = [np.zeros((-(-length // 32) * 32, kv, d)) for _ in range(2)]
    there = np.zeros(out[0].shape[0], dtype=bool)
    for n in range(-(-length // 32)):
        page = int(table[n // per])
        if not 0 <= page < pages:
            continue
        g = memory[page, :, n % per]
        there[32 * n:32 * n + 32] = True
        for o, code, scale in ((out[0], pk, pks), (out[1], pv, pvs)):
            c = g[:, code]
            c = np.stack((c & 15, c >> 4), -1).reshape(kv, 32, d)
            o[32 * n:32 * n + 32] = values(c, g[:, scale]).transpose(1, 0, 2)
    return out[0][:length], out[1][:length], there[:length]


def norm_rotate(x, weight, eps, positions, rotation, rotary, style):
    """x [tokens][heads][d] in binary64; weight: values or None; rotation: [rows][rotary] binary32.  The result rounded to binary32."""
    with np.errstate(all="ignore"):
        y = np.array(x, dtype=np.float64)
        if weight is not None:
            y = y * (1.0 / np.sqrt(np.mean(y * y, axis=-1, keepdims=True) + eps)) * weight
        if rotary:
            held = (positions >= 0) & (positions < rotation.shape[0])
            turn = np.where(held[:, None], rotation[np.where(held, positions, 0)].astype(np.float64), np.nan)[:, None]
            c, s = turn[..., :rotary // 2], turn[..., rotary // 2:]
            i = np.arange(rotary // 2)
            a, b = (i, i + rotary // 2) if style == HALVES else (2 * i, 2 * i + 1)
            ya, yb = y[..., a].copy(), y[..., b].copy()
            y[..., a], y[..., b] = ya * c - yb * s, yb * c + ya * s
        return y.astype(np.float32)


def attention(q, k, v, there, start, scale, window):
    """One sequence: q [n][heads][d], k and v [length][kv][d], row i at position start + i.  Returns the outputs, and for error bounds of each output the
    weighted mean of |v|, and of each row the largest sum of |q k| and the largest score (natural units), and how many tokens it sees."""
    n, heads, d = q.shape
    length, kv = k.shape[:2]
    out, spread = np.zeros((n, heads, d)), np.zeros((n, heads, d))
    most, top, count = np.zeros((n, heads)), np.zeros((n, heads)), np.zeros(n, dtype=int)
    t = np.arange(length)
    with np.errstate(all="ignore"):
        for i in range(n):
            p = start + i
            seen = there & (t <= p)
            if window:
                seen &= t > p - window
            count[i] = seen.sum()
            if not count[i]:
                continue
            for h in range(heads):
                kk, vv = k[seen, h // (heads // kv)], v[seen, h // (heads // kv)]
                z = kk @ q[i, h] * scale
                w = np.exp(z - (np.nan if np.isnan(z).any() else z.max()))
                w = w / w.sum()
                out[i, h] = w @ vv
                spread[i, h] = w @ np.abs(vv)
                most[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * scale
                top[i, h] = np.abs(z).max()
    return out, spread, most, top, count
