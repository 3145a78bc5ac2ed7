"""The cache in 4 bits on the GPU against the binary64 oracle: appending to it, attention over it, copies of its pages."""
import numpy as np
import pytest
import torch

from cache_fp4_cases import Sequences, attention_oracle, worst
from oracle import block_scale as bs
from oracle import cache_fp4 as oc
from paper_2511_10909_amd import binding as mm

pytestmark = pytest.mark.gpu
HALF_STEP = {mm.BF16: 2.0 ** -8, mm.FP16: 2.0 ** -11}             # eps / 2 of the type
GUARD = 0xA5


def dev(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view({2: np.int16, 4: np.int32, 1: np.uint8}[a.dtype.itemsize])).cuda()


def guarded(rows, stride):
    return torch.full((rows, stride), int(np.int16(-0x5A5B)), dtype=torch.int16, device="cuda")


# ---- append -------------------------------------------------------------------------------

def angles(rows, rotary, seed=0):
    a = np.arange(rows)[:, None] * 10000.0 ** (-np.arange(0, rotary, 2) / rotary)
    return np.concatenate([np.cos(a), np.sin(a)], 1).astype(np.float32)


def run_append(seqs, heads, t, x, q_weight=None, k_weight=None, weight_type=None, rotary=0, style=mm.ROTATE_HALVES, rows=None, rule=bs.FLOOR, eps=1e-6,
               pad=0, in_place=False, parts="qkv", stream=None, want_values=True, **more):
    """x: bit patterns [tokens][heads + 2 kv][d].  Compares everything that the call may write with the oracle, bit for bit."""
    d, kv, tokens = seqs.dim, seqs.kv, seqs.tokens
    has_q, has_kv = "q" in parts, "k" in parts
    stride = (heads + 2 * kv) * d + pad
    wide = np.full((tokens + 1, stride), 0x7E55, dtype=np.uint16)
    wide[:tokens, :stride - pad] = x.reshape(tokens, -1)
    dx = dev(wide)
    at = dx.data_ptr()
    q, k, v = at, at + 2 * heads * d, at + 2 * (heads + kv) * d
    out_stride = stride if in_place else heads * d + 8
    out = None if in_place else guarded(tokens + 1, out_stride)
    values = [guarded(tokens + 1, kv * d) for _ in range(2)]
    cache = dev(seqs.memory)
    rot = angles(seqs.columns * seqs.page if rows is None else rows, rotary) if rotary else None
    drot = None if rot is None else torch.from_numpy(rot).cuda()
    dw = [None if w is None else dev(w) for w in (q_weight, k_weight)]
    lengths, table, begins = dev(np.array(seqs.lengths, dtype=np.int32)), dev(seqs.table), dev(seqs.begins)
    torch.cuda.synchronize()
    mm.cache_append_fp4(q if has_q else None, k if has_kv else None, v if has_kv else None, (q if in_place else out) if has_q else None, cache, table, lengths, begins, t,
                        **seqs.shape(heads if has_q else 0, **more), q_weight=dw[0], k_weight=dw[1], weight_type=weight_type, rotation=drot, rotary_dim=rotary,
                        rotation_rows=0 if rot is None else rot.shape[0], rotation_style=style, scale_rule=rule, eps=eps, q_stride=stride, k_stride=stride, v_stride=stride,
                        q_out_stride=out_stride, k_values=values[0] if has_kv and want_values else None, v_values=values[1] if has_kv and want_values else None, stream=stream)
    torch.cuda.synchronize()

    most = more.get("max_tokens", max(seqs.fresh + [0]))
    val = bs.values_of(x, t)
    wt = t if weight_type is None else weight_type
    wq, wk = (None if w is None else bs.values_of(w, wt) for w in (q_weight, k_weight))
    memory = seqs.memory.copy()
    got_q = (dx if in_place else out).cpu().numpy().view(np.uint16)
    got_q = got_q[:, :heads * d]
    got_values = [y.cpu().numpy().view(np.uint16) for y in values]
    written = np.zeros(tokens + 1, dtype=bool)
    for s, n in enumerate(seqs.fresh):
        length = min(max(seqs.lengths[s], 0), seqs.columns * seqs.page)
        first, m = int(seqs.begins[s]), min(n, most)
        if m == 0:
            continue
        rows_of = slice(first, first + m)
        written[rows_of] = True
        pos = np.arange(length - n, length - n + m)
        table_of = np.zeros((0, 16), np.float32) if rot is None else rot
        if has_q:
            y = bs.bits_of(oc.norm_rotate(val[rows_of, :heads], wq, eps, pos, table_of, rotary, style), t).reshape(m, heads * d)
            same = got_q[rows_of] == y
            same |= np.isnan(bs.values_of(got_q[rows_of], t)) & np.isnan(bs.values_of(y, t))
            assert same.all(), (s, np.argwhere(~same)[:5])
        if has_kv:
            kc, ks, kvals = oc.quantize(oc.norm_rotate(val[rows_of, heads:heads + kv], wk, eps, pos, table_of, rotary, style), rule)
            vc, vs, vvals = oc.quantize(val[rows_of, heads + kv:].astype(np.float32), rule)
            for i in range(m):
                if pos[i] >= 0:
                    oc.write(memory, seqs.table[s], seqs.page, int(pos[i]), kc[i], ks[i], vc[i], vs[i])
            if want_values:
                for g, w in zip(got_values, (kvals, vvals)):
                    w = w.reshape(m, kv * d)
                    y = bs.values_of(g[rows_of], t)
                    assert ((y == w) | (np.isnan(y) & np.isnan(w))).all()
    assert np.array_equal(cache.cpu().numpy(), memory)
    guard = np.uint16(0xA5A5)
    if has_q and not in_place:
        assert (got_q[~written] == guard).all() and (out.cpu().numpy().view(np.uint16)[:, heads * d:] == guard).all()
    if has_q and in_place:
        whole = dx.cpu().numpy().view(np.uint16)
        assert np.array_equal(whole[:, heads * d:], wide[:, heads * d:]) and np.array_equal(got_q[~written], wide[~written, :heads * d])
    for g in got_values:
        assert (g[~written] == guard).all() and (has_kv and want_values or (g == guard).all())
    return memory


def inputs(seqs, heads, t):
    return bs.bits_of(seqs.heads(seqs.tokens, heads + 2 * seqs.kv), t)


def weights(seqs, t):
    return [bs.bits_of((1 + 0.2 * seqs.rng.standard_normal(seqs.dim)).astype(np.float32), t) for _ in range(2)]


@pytest.mark.parametrize("t", [mm.BF16, mm.FP16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("start", [0, 1, 3, 4, 6, 31, 61])
@pytest.mark.parametrize("fresh", [1, 2, 5, 9, 40])
def test_append_lengths(t, d, start, fresh):
    seqs = Sequences(start + 100 * fresh, [fresh], [start + fresh], d, 2, 32)
    qw, kw = weights(seqs, t)
    run_append(seqs, 5, t, inputs(seqs, 5, t), qw, kw, rotary=d)


@pytest.mark.parametrize("t,wt", [(mm.BF16, mm.BF16), (mm.BF16, mm.FP32), (mm.FP16, mm.FP16), (mm.FP16, mm.FP32)])
@pytest.mark.parametrize("d,rotary,style", [(128, 128, 0), (128, 64, 0), (128, 16, 1), (128, 0, 0), (64, 64, 1), (64, 32, 0), (64, 16, 0), (64, 48, 1)])
@pytest.mark.parametrize("rule", [bs.FLOOR, bs.FIT])
def test_append_norms_and_rotations(t, wt, d, rotary, style, rule):
    seqs = Sequences(d + rotary, [3, 1, 8, 17], [40, 1, 100, 17], d, 3, 64)
    qw, kw = weights(seqs, wt)
    x = inputs(seqs, 7, t)
    run_append(seqs, 7, t, x, qw, kw, weight_type=wt, rotary=rotary, style=style, rule=rule, pad=8)
    run_append(seqs, 7, t, x, None, kw, weight_type=wt, rotary=rotary, style=style, rule=rule, eps=0.0, in_place=True)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [32, 96, 256])
def test_append_many_sequences(d, page):
    rng = np.random.default_rng(page)
    fresh = [int(x) for x in rng.integers(0, 12, 30)]
    seqs = Sequences(d, fresh, [f + int(x) for f, x in zip(fresh, rng.integers(0, 400, 30))], d, 2, page)
    qw, kw = weights(seqs, mm.BF16)
    run_append(seqs, 2, mm.BF16, inputs(seqs, 2, mm.BF16), qw, kw, rotary=d, want_values=False)


@pytest.mark.parametrize("parts", ["q", "kv"])
def test_append_of_queries_or_keys_alone(parts):
    seqs = Sequences(5, [4, 1], [9, 70], 128, 2, 64)
    qw, kw = weights(seqs, mm.FP16)
    run_append(seqs, 4, mm.FP16, inputs(seqs, 4, mm.FP16), qw, kw, rotary=128, parts=parts)


@pytest.mark.parametrize("d", [64, 128])
def test_append_takes_any_numbers(d):
    """Zeros, infinities, NaN, blocks that saturate, vanish or are subnormal."""
    seqs = Sequences(8, [10, 3], [10, 35], d, 2, 32)
    x = seqs.heads(13, 3 + 4)
    x[1], x[2, :, 5], x[3, :, d // 2] = 0, np.inf, np.nan
    x[4], x[5], x[6] = x[4] * np.float32(1e30), x[5] * np.float32(1e-30), x[6] * np.float32(1e-39)
    x[7, :, :32], x[8, :, ::2], x[9] = 0, -0.0, 60000.0
    for rule in (bs.FLOOR, bs.FIT):
        for t in (mm.BF16, mm.FP16):
            bits = bs.bits_of(x, t)
            qw, kw = weights(seqs, t)
            run_append(seqs, 3, t, bits, qw, kw, rotary=d, rule=rule)
            run_append(seqs, 3, t, bits, None, None, rule=rule, eps=0.0)


def test_append_where_tables_and_lengths_say_otherwise():
    """Pages that are none, lengths below what comes and above what the table holds, more tokens than max_tokens, positions without an angle."""
    seqs = Sequences(3, [5, 4, 6, 2, 3], [70, 40, 4, 33, 3], 128, 2, 32)
    seqs.table[0, 2], seqs.table[1, 1] = seqs.pages, -7
    seqs.table[3, 1] = 2 ** 31 - 1
    seqs.lengths[4] = 10 ** 6
    seqs.table[4, :] = [x for x in range(seqs.pages) if x not in seqs.table][:1] + [-1] * (seqs.columns - 1)
    qw, kw = weights(seqs, mm.BF16)
    x = inputs(seqs, 2, mm.BF16)
    run_append(seqs, 2, mm.BF16, x, qw, kw, rotary=128)
    run_append(seqs, 2, mm.BF16, x, qw, kw, rotary=128, rows=67)
    run_append(seqs, 2, mm.BF16, x, qw, kw, rotary=64, max_tokens=3)
    seqs.lengths[2] = -5
    run_append(seqs, 2, mm.BF16, x, qw, kw, rotary=64)


# ---- attention ------------------------------------------------------------------------------

def run_attention(seqs, heads, t, q=None, window=0, scale=None, pad=0, in_place=False, max_length=None, stream=None, **more):
    """Outputs within the derived bounds; rows of no sequence and the room between rows stay as they were."""
    d, tokens = seqs.dim, seqs.tokens
    scale = d ** -0.5 if scale is None else scale
    q = bs.bits_of(1.5 * seqs.heads(tokens, heads), t) if q is None else q
    stride = heads * d + pad
    wide = np.full((tokens + 1, stride), 0x7E55, dtype=np.uint16)
    wide[:tokens, :heads * d] = q.reshape(tokens, -1)
    dq = dev(wide)
    out = dq if in_place else guarded(tokens + 1, stride)
    shape = seqs.shape(heads, **more)
    longest = max(seqs.lengths + [1]) if max_length is None else max_length
    size = mm.attention_fp4_workspace(t, max_length=longest, window=window, **shape)
    ws = torch.full((size + 256,), GUARD, dtype=torch.uint8, device="cuda")
    arrays = [dev(seqs.memory), dev(seqs.table), dev(np.array(seqs.lengths, dtype=np.int32)), dev(seqs.begins)]
    torch.cuda.synchronize()
    mm.attention_fp4(dq, out, *arrays, ws if size else None, t, **shape, max_length=longest, scale=scale, window=window, q_stride=stride, out_stride=stride,
                     workspace_bytes=size, stream=stream)
    torch.cuda.synchronize()
    assert (ws[size:] == GUARD).all()
    got = out.cpu().numpy().view(np.uint16)
    want, room, mine = attention_oracle(seqs, bs.values_of(q, t), heads, scale, window, shape["max_tokens"])
    y = bs.values_of(got[:tokens, :heads * d], t).reshape(tokens, heads, d)
    off = worst(y[mine], want[mine], room[mine], HALF_STEP[t])
    assert off <= 1.0, off
    before = wide if in_place else np.full_like(wide, 0xA5A5)
    assert np.array_equal(got[:, heads * d:], before[:, heads * d:]) and np.array_equal(got[:tokens][~mine], before[:tokens][~mine]) and np.array_equal(got[tokens], before[tokens])
    return got


@pytest.mark.parametrize("t", [mm.BF16, mm.FP16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", [1, 3, 8, 16, 21])
@pytest.mark.parametrize("length", [1, 2, 31, 32, 33, 64, 65, 300, 1025])
def test_attention_of_one_token(t, d, group, length):
    seqs = Sequences(length + group, [1], [length], d, 2, 32).fill()
    run_attention(seqs, 2 * group, t)


@pytest.mark.parametrize("t", [mm.BF16, mm.FP16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group,fresh,length", [(4, 2, 2), (4, 5, 40), (1, 16, 16), (1, 17, 300), (8, 5, 77), (2, 33, 65), (4, 40, 40), (5, 31, 130), (4, 70, 321), (1, 257, 257), (8, 33, 500)])
@pytest.mark.parametrize("window", [0, 7, 64])
def test_attention_of_several_tokens(t, d, group, fresh, length, window):
    seqs = Sequences(length + fresh, [fresh], [length], d, 2, 64).fill()
    run_attention(seqs, 2 * group, t, window=window, pad=8)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [32, 96, 256])
@pytest.mark.parametrize("window", [0, 1, 50, 1000])
@pytest.mark.parametrize("most", [1, 6, 60])
def test_attention_of_many_sequences(d, page, window, most):
    rng = np.random.default_rng(page + window)
    fresh = [int(x) for x in rng.integers(0, most + 1, 9)]
    seqs = Sequences(page, fresh, [f + int(x) for f, x in zip(fresh, rng.integers(0, 700, 9))], d, 2, page).fill()
    run_attention(seqs, 8, mm.BF16, window=window, in_place=True)


@pytest.mark.parametrize("d,fresh,length,window", [(128, 1, 9000, 0), (64, 1, 20000, 0), (128, 3, 9000, 5000), (64, 40, 6000, 0), (128, 130, 3000, 0), (128, 20, 3000, 100)])
def test_attention_over_long_caches(d, fresh, length, window):
    seqs = Sequences(length, [fresh], [length], d, 1, 128).fill()
    for t in (mm.BF16, mm.FP16):
        run_attention(seqs, 4, t, window=window)
    # what the host says of the length decides over the launch, not over the result
    run_attention(seqs, 4, mm.FP16, window=window, max_length=1)
    run_attention(seqs, 4, mm.FP16, window=window, max_length=length * 20)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("empty", [105, 215])
@pytest.mark.parametrize("window", [0, 40, 1300])
def test_attention_of_chunks_among_many_sequences(d, empty, window):
    """Chunks over long caches in a batch whose other sequences bring nothing: wavefronts of two and three tiles of rows, in one part and in two."""
    def alter(s, k, v):
        if s == 1:
            v[3, 0], k[9, 1, 3], v[-1, 1, :32] = np.nan, np.nan, np.inf
    fresh, lengths = [48, 45, 17, 1, 48] + [0] * empty, [3000, 800, 1500, 900, 2530] + [0] * empty
    seqs = Sequences(empty, fresh, lengths, d, 2, 64).fill(alter)
    seqs.table[4, 1] = -1
    shape = seqs.shape(8)
    # (two parts; the plan counts a window's tokens where they are fewer)
    size = mm.attention_fp4_workspace(mm.BF16, max_length=3000, window=window, **shape)
    assert size == (2 * seqs.tokens * 8 * (d + 2) * 4 if window == 0 else 0)
    run_attention(seqs, 8, mm.BF16, window=window, pad=8)
    run_attention(seqs, 8, mm.FP16, window=window, in_place=True, max_length=100000)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sequences", [2, 63, 64, 65])
def test_attention_in_any_order_of_lengths(d, sequences):
    """The longest sequences' workgroups start first: equal lengths, sequences that bring nothing, lengths that are none."""
    rng = np.random.default_rng(sequences)
    fresh = [int(x) for x in rng.integers(0, 25, sequences)]
    fresh[0], fresh[-1] = 25, 20
    lengths = [f + 40 * int(x) for f, x in zip(fresh, rng.integers(0, 4, sequences))]
    # (a sequence whose length will say more than was written has its pages full: what other bytes mean as scales is nowhere said)
    lengths[sequences // 3] = -(-max(lengths[sequences // 3], 1) // 32) * 32
    seqs = Sequences(sequences, fresh, lengths, d, 1, 32).fill()
    seqs.lengths[sequences // 2], seqs.lengths[sequences // 3] = -5, 10 ** 6
    run_attention(seqs, 3, mm.FP16, max_length=300)
    run_attention(seqs, 3, mm.BF16, max_length=1)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fresh", [1, 6, 50])
def test_attention_does_not_see_what_is_not_there(d, fresh):
    """Keys and values that are NaN: outputs are NaN where a row sees them (values: in their block alone), and nowhere else."""
    def alter(s, k, v):
        n = k.shape[0]
        if s == 0:
            k[n - 1, 0, 3], v[n - 1, 1, 40] = np.nan, np.inf            # the last token: seen by the last row alone
        if s == 1:
            v[5, 0, :32], v[n // 2, 1, d - 1] = np.nan, np.nan
            k[7, 1] = np.nan
        if s == 2:
            v[n - 3], k[n - 3] = 0, 0
    seqs = Sequences(fresh, [fresh] * 4, [fresh + 70, fresh + 40, fresh + 100, fresh], d, 2, 32).fill(alter)
    run_attention(seqs, 8, mm.BF16)
    run_attention(seqs, 8, mm.FP16, window=20)


@pytest.mark.parametrize("fresh", [1, 30])
def test_attention_where_tables_and_lengths_say_otherwise(fresh):
    """Pages that are none are not there; rows that see no token give zeros; more tokens than max_tokens."""
    seqs = Sequences(fresh, [fresh, fresh, fresh, 3, fresh], [150, 200, 90, 1, fresh + 3], 128, 2, 32).fill()
    seqs.table[0, 1], seqs.table[1, 0], seqs.table[1, 3] = seqs.pages, -1, 2 ** 31 - 1
    seqs.table[2, :] = -2
    run_attention(seqs, 6, mm.BF16)
    run_attention(seqs, 6, mm.BF16, window=33)
    run_attention(seqs, 6, mm.BF16, max_tokens=2)
    seqs.lengths[0], seqs.lengths[4] = -3, 0
    run_attention(seqs, 6, mm.FP16)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_of_extreme_queries(d):
    """Scores of thousands, of nearly nothing, all alike; NaN and infinite queries touch their own row alone."""
    seqs = Sequences(d, [8], [200], d, 1, 64).fill()
    q = 1.5 * seqs.heads(8, 4)
    q[0] *= 300
    q[1] *= 1e-4
    q[2] = 0
    run_attention(seqs, 4, mm.BF16, bs.bits_of(q, mm.BF16))
    run_attention(seqs, 4, mm.FP16, bs.bits_of(q, mm.FP16), scale=3.0)
    q[5, 1, 4] = np.nan
    q[7, :, 0] = np.inf
    got = run_attention(seqs, 4, mm.FP16, bs.bits_of(np.where(np.isinf(q), np.nan, q), mm.FP16))
    assert got is not None


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fresh,length", [(1, 1), (1, 2100), (5, 70), (70, 70), (70, 2200)])
@pytest.mark.parametrize("magnitude", [2.0 ** 12, 2.0 ** 22, 2.0 ** 24, 2.0 ** 31, 2.0 ** 70, 2.0 ** 127])
@pytest.mark.parametrize("sign", [-1, 1])
def test_attention_of_equal_and_far_scores(d, fresh, length, magnitude, sign):
    """Scores up to the largest numbers there are.  Where all of a row's tokens have the same, the output is their values' mean; a token whose key is twice as
    large (rows 70 on of the second head see it) has all the weight, or none where scores are negative.

    One element of a key is not zero, so that scores are exact.  The weights of equal scores are one and the same number, in all parts of a row: what is left are
    binary32 sums of `count` values and the join's, (count + 64) 2^-23 of the values' mean magnitude.  The larger key's scores differ by 2^11 and more in units of log2."""
    big = length - fresh // 2 - 1

    def alter(s, k, v):
        k[:] = 0
        k[..., 5] = 1
        k[big, 1, 5] = 2 if magnitude < 2.0 ** 127 else 1
    seqs = Sequences(fresh + d, [fresh], [length], d, 2, 32).fill(alter)
    scale = np.log(2.0) * (1 - 2.0 ** -20)
    q = np.zeros((fresh, 4, d), dtype=np.float32)
    q[..., 5] = sign * 1.9921875 * magnitude
    out = guarded(fresh, 4 * d)
    arrays = [dev(bs.bits_of(q, mm.BF16).reshape(fresh, -1)), out, dev(seqs.memory), dev(seqs.table), dev(np.array(seqs.lengths, dtype=np.int32)), dev(seqs.begins)]
    shape = seqs.shape(4)
    size = mm.attention_fp4_workspace(mm.BF16, max_length=length, **shape)
    assert (size > 0) == (length > 2000)
    ws = torch.empty(size + 16, dtype=torch.uint8, device="cuda")
    mm.attention_fp4(*arrays, ws if size else None, mm.BF16, **shape, max_length=length, scale=float(scale), workspace_bytes=size)
    torch.cuda.synchronize()
    got = bs.values_of(out.cpu().numpy().view(np.uint16), mm.BF16).reshape(fresh, 2, 2, d)
    _, v, _ = oc.read(seqs.memory, seqs.table[0], seqs.page, length, d)
    for i in range(fresh):
        seen = length - fresh + i + 1
        for h in range(2):
            use = np.arange(seen)
            if h == 1 and seen > big and magnitude < 2.0 ** 127 and seen > 1:
                use = use[use == big] if sign > 0 else use[use != big]
            want, most = v[use, h].mean(0), np.abs(v[use, h]).mean(0)
            room = (seen + 64) * 2.0 ** -23 * most
            assert (np.abs(got[i, h] - want) <= room + 2.0 ** -8 * (np.abs(want) + room)).all(), (i, h)


def test_attention_past_32_bits_of_bytes():
    """A sequence whose pages lie beyond 4 GiB of the cache."""
    seqs = Sequences(1, [2], [300], 128, 8, 256, spare=0).fill()
    per = mm.cache_page_bytes(128, 8, 256)
    pages = (5 << 30) // per
    cache = torch.empty((pages, 8, 8, 34 * 128), dtype=torch.uint8, device="cuda")
    high = [pages - 1, pages - 9]
    table = seqs.table.copy()
    for i, p in enumerate(high):
        cache[p] = torch.from_numpy(seqs.memory[seqs.table[0, i]]).cuda()
        table[0, i] = p
    q = bs.bits_of(seqs.heads(2, 8), mm.BF16)
    dq, out = dev(q), guarded(2, 1024)
    shape = seqs.shape(8, pages=pages)
    size = mm.attention_fp4_workspace(mm.BF16, max_length=300, **shape)
    ws = torch.empty(max(size, 16), dtype=torch.uint8, device="cuda")
    lengths, begins, dtable = dev(np.array([300], dtype=np.int32)), dev(seqs.begins), dev(table)
    mm.attention_fp4(dq, out, cache, dtable, lengths, begins, ws, mm.BF16, **shape, max_length=300, scale=0.1, workspace_bytes=size)
    torch.cuda.synchronize()
    want, room, _ = attention_oracle(seqs, bs.values_of(q, mm.BF16), 8, 0.1)
    assert worst(bs.values_of(out.cpu().numpy().view(np.uint16), mm.BF16).reshape(2, 8, 128), want, room, HALF_STEP[mm.BF16]) <= 1.0
    # and a token appended there
    kv = bs.bits_of(seqs.heads(2, 16), mm.BF16)
    dkv = dev(kv)
    mm.cache_append_fp4(None, dkv.data_ptr(), dkv.data_ptr() + 2 * 8 * 128, None, cache, dtable, lengths, begins, mm.BF16, **seqs.shape(0, pages=pages),
                        k_stride=16 * 128, v_stride=16 * 128)
    torch.cuda.synchronize()
    val = bs.values_of(kv, mm.BF16)
    memory, at = seqs.memory.copy(), seqs.table[0]
    for i in range(2):
        (kc, ks, _), (vc, vs, _) = oc.quantize(val[i, :8], bs.FLOOR), oc.quantize(val[i, 8:], bs.FLOOR)
        oc.write(memory, at, 256, 298 + i, kc, ks, vc, vs)
    for i, p in enumerate(high):
        assert np.array_equal(cache[p].cpu().numpy(), memory[at[i]])


# ---- copies ---------------------------------------------------------------------------------

@pytest.mark.parametrize("page_bytes", [16, 48, 4096, 16384, 16400, 34816, 69632])
@pytest.mark.parametrize("layers,gap", [(1, 0), (3, 32)])
def test_copies(page_bytes, layers, gap):
    rng = np.random.default_rng(page_bytes)
    pages = 23
    memory = rng.integers(0, 256, layers * (pages * page_bytes + gap)).astype(np.uint8)
    order = rng.permutation(pages)
    moves = [(order[0], order[1]), (order[0], order[2]), (order[3], order[4]), (order[5], order[5]), (order[6], order[7])]
    d = torch.from_numpy(memory.copy()).cuda()
    torch.cuda.synchronize()
    mm.cache_copy_pages(d, torch.tensor(np.array(moves), dtype=torch.int32), pages, page_bytes, layers, pages * page_bytes + gap if gap else 0)
    torch.cuda.synchronize()
    want = memory.reshape(layers, -1)
    body = want[:, :pages * page_bytes].reshape(layers, pages, page_bytes)
    new = body.copy()
    for a, b in moves:
        new[:, b] = body[:, a]
    want = np.concatenate([new.reshape(layers, -1), want[:, pages * page_bytes:]], 1)
    assert np.array_equal(d.cpu().numpy().reshape(layers, -1), want)


def test_more_copies_than_one_launch_takes():
    rng = np.random.default_rng(0)
    pages = 3001
    memory = rng.integers(0, 256, (2, pages, 208)).astype(np.uint8)
    order = rng.permutation(pages)[:3000].reshape(-1, 2)
    order[7, 1] = order[7, 0]
    d = torch.from_numpy(memory).cuda()
    mm.cache_copy_pages(d, torch.tensor(order, dtype=torch.int32), pages, 208, 2)
    torch.cuda.synchronize()
    want = memory.copy()
    want[:, order[:, 1]] = memory[:, order[:, 0]]
    assert np.array_equal(d.cpu().numpy(), want)
