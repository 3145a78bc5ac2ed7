"""Sequences in a cache of 4 bits for tests: pages in no order, memory that holds anything where no token lies, and the binary64 oracle's side of a call."""
import numpy as np

from oracle import block_scale as bs
from oracle import cache_fp4 as oc


class Sequences:
    """`fresh` tokens of each sequence come with a call, `lengths` are in the cache after it."""

    def __init__(self, seed, fresh, lengths, dim, kv, page, spare=2, extra_columns=1):
        self.rng = np.random.default_rng(seed)
        self.fresh, self.lengths, self.dim, self.kv, self.page = fresh, lengths, dim, kv, page
        counts = [-(-max(n, 0) // page) for n in lengths]
        self.pages = sum(counts) + spare
        self.columns = max(counts + [1]) + extra_columns
        order = self.rng.permutation(self.pages)
        self.table = np.full((len(fresh), self.columns), -1, dtype=np.int32)
        at = 0
        for s, c in enumerate(counts):
            self.table[s, :c] = order[at:at + c]
            at += c
        self.begins = np.concatenate(([0], np.cumsum(fresh))).astype(np.int32)
        self.tokens = int(self.begins[-1])
        # what nobody wrote: any bytes, NaN scales and codes that no cache holds among them
        self.memory = self.rng.integers(0, 256, (self.pages, kv, page // 32, 34 * dim)).astype(np.uint8)

    def shape(self, heads, **more):
        return dict(dict(dim=self.dim, heads=heads, kv_heads=self.kv, page_tokens=self.page, pages=self.pages, sequences=len(self.fresh),
                         table_stride=self.columns, tokens=self.tokens, max_tokens=max(self.fresh + [0])), **more)

    def heads(self, tokens, heads, std=1.0):
        x = self.rng.standard_normal((tokens, heads, self.dim)) * np.exp(0.5 * self.rng.standard_normal((tokens, heads, 1))) * std
        x[..., ::29] *= 4
        return x.astype(np.float32)

    def fill(self, alter=None):
        """Every token of every sequence as keys and values of ordinary size; alter(s, k, v) may change them first."""
        for s, n in enumerate(self.lengths):
            if n <= 0:
                continue
            k, v = self.heads(n, self.kv), self.heads(n, self.kv, 0.3)
            if alter:
                alter(s, k, v)
            kc, ks, _ = oc.quantize(k, bs.FLOOR)
            vc, vs, _ = oc.quantize(v, bs.FLOOR)
            for t in range(n):
                oc.write(self.memory, self.table[s], self.page, t, kc[t], ks[t], vc[t], vs[t])
        return self


def attention_oracle(seqs, q, heads, scale, window=0, max_tokens=None):
    """q: values [tokens][heads][dim].  (outputs, absolute error allowed before the output's own rounding, rows that belong to a sequence).

    The kernel's sums: a score is a sum of dim products in binary32 (each step off by at most 2^-23 of the sum of magnitudes), times the
    scale in units of log2, minus the maximum, plus a shift of at most ten (steps of 2^-24 of numbers up to their magnitude + 10), its exponential within
    2^-22; the weight, held times 2^4 or more of the largest, is rounded to FP16: 2^-11 relative, and below its normal numbers half a step of 2^-24, which is 2^-29 of the
    largest weight and so of their sum; sums over tokens in binary32."""
    d = seqs.dim
    want, room = np.zeros((seqs.tokens, heads, d)), np.zeros((seqs.tokens, heads, d))
    mine = np.zeros(seqs.tokens, dtype=bool)
    for s, n in enumerate(seqs.fresh):
        m = n if max_tokens is None else min(n, max_tokens)
        at = slice(seqs.begins[s], seqs.begins[s] + m)
        mine[at] = True
        length = min(max(seqs.lengths[s], 0), seqs.columns * seqs.page)
        k, v, there = oc.read(seqs.memory, seqs.table[s], seqs.page, length, d)
        o, spread, most, top, count = oc.attention(q[at], k, v, there, length - n, scale, window)
        log2e = 1.4426950408889634
        score = (d * 2.0 ** -23 * most + 2.0 ** -23 * (2 * top + 10)) * log2e * 2           # of a score and of the row's maximum, in log2
        weight = np.expm1(score * np.log(2)) + 2.0 ** -22
        want[at] = o
        room[at] = spread * (2.0 ** -11 + 2 * weight[..., None] + (count[:, None, None] + 64) * 2.0 ** -23) + count[:, None, None] * 2.0 ** -29 * (np.nanmax(np.abs(v), initial=0.0))
    return want, room, mine


def worst(got, want, room, half_step):
    """The largest error of outputs over what is allowed: room, and half a step of the output's type (half_step relative, at least 2^-25 as FP16 has at its end);
    NaN in the same places."""
    nan = np.isnan(want)
    assert np.array_equal(nan, np.isnan(got))
    got, want, room = got[~nan], want[~nan], room[~nan]
    if not got.size:
        return 0.0
    allowed = room + half_step * (np.abs(want) + room) + 2.0 ** -25
    return float((np.abs(got - want) / allowed).max())
