"""Weights of scores that are equal, or a few units apart, whatever their size, and of scores that are infinite: attention over a cache whose scores are known exactly."""
import numpy as np
import pytest
import torch

from cache_fp4_cases import Sequences, worst
from oracle import block_scale as bs
from oracle import cache_fp4 as oc
from paper_2511_10909_amd import binding as mm

pytestmark = pytest.mark.gpu
HALF_STEP = {mm.BF16: 2.0 ** -8, mm.FP16: 2.0 ** -11}


def dev(a):
    a = np.ascontiguousarray(a)
    return torch.from_numpy(a.view({2: np.int16, 4: np.int32, 1: np.uint8}[a.dtype.itemsize])).cuda()


def attend(seqs, q, t, scale):
    """q: values [tokens][heads][dim] that the type holds; the outputs as values."""
    tokens, heads, d = q.shape
    bits = bs.bits_of(q, t)
    assert np.array_equal(bs.values_of(bits, t), q)                  # (infinities among them)
    longest, shape = max(seqs.lengths), seqs.shape(heads)
    size = mm.attention_fp4_workspace(t, max_length=longest, **shape)
    ws = torch.empty(size + 16, dtype=torch.uint8, device="cuda")
    out = torch.zeros((tokens, heads * d), dtype=torch.int16, device="cuda")
    arrays = [dev(bits.reshape(tokens, -1)), out, dev(seqs.memory), dev(seqs.table), dev(np.array(seqs.lengths, dtype=np.int32)), dev(seqs.begins)]
    torch.cuda.synchronize()
    mm.attention_fp4(*arrays, ws if size else None, t, **shape, max_length=longest, scale=float(scale), workspace_bytes=size)
    torch.cuda.synchronize()
    return bs.values_of(out.cpu().numpy().view(np.uint16), t).reshape(tokens, heads, d)


# one token: eight wavefronts share the tokens, in one part and in several; drafts: four tiles; a chunk: rows over wavefronts
FORMS = [(1, 512), (1, 512 * 32), (20, 512), (70, 512), (70, 4096)]


@pytest.mark.parametrize("t", [mm.BF16, mm.FP16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fresh,length", FORMS)
@pytest.mark.parametrize("power", [10, 13, 15, 17, 19, 20, 21, 22, 23])
def test_equal_scores_weigh_the_same(t, d, fresh, length, power):
    """All tokens have one score x (one element of a key is not zero), around 2^power in units of log2, the values 1 in a row's first tokens and -1 in later ones.  Weights are one
    and the same number, so that the output is the values' mean: what is left are binary32 sums of `seen` values and the joins', (seen + 64) 2^-23."""
    first = 256 if fresh == 1 else 32              # each wavefront's first granule, or the first of all

    def alter(s, k, v):
        k[:] = 0
        k[..., 5] = 1
        v[:first], v[first:] = 1, -1
    seqs = Sequences(power, [fresh], [length], d, 2, 64).fill(alter)
    q = np.zeros((fresh, 8, d), dtype=np.float32)
    most = 2.0 ** power if t == mm.BF16 else 2.0 ** min(power, 14)
    for h in range(8):
        q[:, h, 5] = most * (1 + 15 * h / 128)
    got = attend(seqs, q, t, 0.7 * 2.0 ** power / most)
    for i in range(fresh):
        seen = length - fresh + i + 1
        want = (first - (seen - first)) / seen
        room = (seen + 64) * 2.0 ** -23
        assert (np.abs(got[i] - want) <= room + HALF_STEP[t] * (abs(want) + room)).all(), (i, np.abs(got[i] - want).max(), room)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fresh,length", FORMS)
@pytest.mark.parametrize("around", [-2.0 ** 22, 2.0 ** 13, 2.0 ** 21, 2.0 ** 22, 2.0 ** 23])
def test_a_score_a_little_larger_between_equal_ones(d, fresh, length, around):
    """All tokens but one have the score x, that one x + 8, x a whole number whose size in units of log2 is just below `around`.  Values are 1 before it, -1 behind.

    Scores are whole numbers below 2^24, exact in binary32.  Weights are 2^(c (s - m)) with c = scale log2(e) in binary32; what may be off are their exponents (sums in binary32 of
    at most 64: 2^-19) and the exponential (2^-22), together 2^-18, in each of two factors, and FP16's rounding of 2^-11; then binary32 sums."""
    at = 256 if fresh == 1 else 100

    def alter(s, k, v):
        k[:] = 0
        k[..., 1:4], k[at, :, 4] = 1, 1
        v[:at], v[at:] = 1, -1
    seqs = Sequences(d, [fresh], [length], d, 2, 64).fill(alter)
    c = np.float64(np.float32(0.5 * 1.4426950408889634))
    # x in three numbers of eight bits each; x c is up to 4 below `around`, so that the larger score's lies beyond it
    x, parts = int(np.floor(around / c - 3)), []
    for unit in (65536, 256, 1):
        parts.append(x // unit * unit)
        x -= parts[-1]
    q = np.zeros((fresh, 8, d), dtype=np.float32)
    for i, p in enumerate(parts):
        q[..., 1 + i] = p
    q[..., 4] = 8
    got = attend(seqs, q, mm.BF16, 0.5)
    for i in range(fresh):
        seen = length - fresh + i + 1
        w = np.full(seen, np.exp2(-8 * c))
        w[at] = 1
        want = (w[:at].sum() - w[at:].sum()) / w.sum()
        room = 2.0 ** -11 + 2.0 ** -17 + (seen + 64) * 2.0 ** -23
        assert (np.abs(got[i] - want) <= room + 2.0 ** -8 * (abs(want) + room)).all(), (i, np.abs(got[i] - want).max(), room)


@pytest.mark.parametrize("fresh,length", FORMS)
@pytest.mark.parametrize("sign", [-1, 1])
@pytest.mark.parametrize("scale", [1e4, 1e30])
def test_scores_that_are_finite_before_they_are_scaled(fresh, length, sign, scale):
    """q . k is a binary32 number, times the scale it is none: equal ones weigh the same, and the largest one has all the weight, or shares none."""
    at = length - fresh // 2 - 1

    def alter(s, k, v):
        k[:] = 0
        k[..., 5] = 1
        k[at, 1, 5] = 2
    seqs = Sequences(fresh, [fresh], [length], 128, 2, 64).fill(alter)
    q = np.zeros((fresh, 4, 128), dtype=np.float32)
    q[..., 5] = sign * 1.5 * 2.0 ** 125
    got = attend(seqs, q, mm.BF16, scale)
    _, v, _ = oc.read(seqs.memory, seqs.table[0], seqs.page, length, 128)
    for i in range(fresh):
        seen = length - fresh + i + 1
        for h in range(4):
            use = np.arange(seen)
            if h >= 2 and seen > at and seen > 1:
                use = use[use == at] if sign > 0 else use[use != at]
            want, most = v[use, h // 2].mean(0), np.abs(v[use, h // 2]).mean(0)
            room = (seen + 64) * 2.0 ** -23 * most
            assert (np.abs(got[i, h] - want) <= room + 2.0 ** -8 * (np.abs(want) + room)).all(), (i, h)


@pytest.mark.parametrize("t", [mm.BF16, mm.FP16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fresh,length", FORMS)
def test_infinite_queries(t, d, fresh, length):
    """Heads of a token, which are rows of one tile: one whose scores are infinities of both signs is NaN, one whose scores are all minus infinity sees nothing, one that has minus
    infinity for every third token weighs the others alone, and the heads beside them are as ever."""
    def alter(s, k, v):
        k[..., 7] = np.where(np.arange(length) % 2, 1, -1)[:, None]
        k[..., 9] = 2
        k[..., 11] = np.where(np.arange(length) % 3, 0, 4)[:, None]
    seqs = Sequences(fresh + d, [fresh], [length], d, 2, 64).fill(alter)
    q = bs.values_of(bs.bits_of(seqs.heads(fresh, 8), t), t).astype(np.float32)
    q[:, [1, 6], 7], q[:, 3, 9], q[:, 4, 7] = np.inf, -np.inf, -np.inf
    k, v, there = oc.read(seqs.memory, seqs.table[0], seqs.page, length, d)
    # (beside large ones elements 7, 9 and 11 may have come to 0: times infinity that is NaN, and so is the row)
    large = k[..., 11] != 0
    assert (k[large][..., 11] >= 2).all() and (large.sum(0) > length // 4).all() and there.all() and ((k[..., 7] > 0).any(0) & (k[..., 7] < 0).any(0)).all()
    lost = np.array([(k[:length - fresh + i + 1, 0, 9] == 0).any() for i in range(fresh)])
    plain = q.copy()
    plain[~np.isfinite(plain)] = 0
    if t == mm.BF16:
        # times four or more this leaves binary32
        q[:, [0, 5], 11], plain[:, [0, 5], 11] = -2.0 ** 127, 0
    got = attend(seqs, q, t, d ** -0.5)
    assert np.isnan(got[:, [1, 4, 6]]).all() and np.isnan(got[lost, 3]).all() and (got[~lost, 3] == 0).all()
    for heads, finite in (([0, 5], ~large if t == mm.BF16 else large | ~large), ([2, 7], large | ~large)):
        for h in heads:
            seen = finite[:, h // 4]
            o, spread, most, top, count = oc.attention(plain[:, [h]].astype(np.float64), k[:, [h // 4]], v[:, [h // 4]], seen, length - fresh, d ** -0.5, 0)
            # the room of the oracle's other users: scores in binary32, weights in FP16, sums over tokens in binary32
            score = (d * 2.0 ** -23 * most + 2.0 ** -23 * (2 * top + 10)) * 1.4426950408889634 * 2
            weight = np.expm1(score * np.log(2)) + 2.0 ** -22
            room = spread * (2.0 ** -11 + 2 * weight[..., None] + (count[:, None, None] + 64) * 2.0 ** -23) + count[:, None, None] * 2.0 ** -29 * np.abs(v).max()
            assert worst(got[:, [h]], o, room, HALF_STEP[t]) <= 1.0, h


@pytest.mark.parametrize("t", [mm.BF16, mm.FP16])
@pytest.mark.parametrize("fresh,length", FORMS)
def test_rows_whose_scores_are_all_one_infinity(t, fresh, length):
    """Minus infinity weighs nothing: a row that has nothing else is zeros; plus infinity makes NaN.  Rows beside them, whose scores are equal, are the values' mean."""
    def alter(s, k, v):
        k[:] = 0
        k[..., 5] = 1
    seqs = Sequences(fresh, [fresh], [length], 64, 2, 64).fill(alter)
    q = np.zeros((fresh, 8, 64), dtype=np.float32)
    q[:, :, 5] = [3, -np.inf, np.inf, -7, np.inf, 0, -np.inf, 300]
    got = attend(seqs, q, t, 1.0)
    assert (got[:, [1, 6]] == 0).all() and np.isnan(got[:, [2, 4]]).all()
    _, v, _ = oc.read(seqs.memory, seqs.table[0], seqs.page, length, 64)
    for i in range(fresh):
        seen = length - fresh + i + 1
        for h in (0, 3, 5, 7):
            want, most = v[:seen, h // 4].mean(0), np.abs(v[:seen, h // 4]).mean(0)
            room = (seen + 64) * 2.0 ** -23 * most
            assert (np.abs(got[i, h] - want) <= room + HALF_STEP[t] * (np.abs(want) + room) + 2.0 ** -25).all(), (i, h)
