// What the attention kernels share: their arguments, the granules that a block of rows sees, and the cache's codes as 16-bit numbers.
#pragma once
#include "cache_fp4.hpp"
#include "fp4_operands.hpp"

namespace mmaemu {

struct AttentionArgs {
    CacheArgs c;
    const void *q;
    void *out;
    float *part;                                   // [split][token][head][D], unnormalised, and behind them
    f32x2 *stat;                                   // [split][token][head]: largest score m, and l, weights relative to 2^(c2 m)
    uint64_t q_stride, out_stride;
    uint32_t heads, group, max_tokens, window, blocks;                 // blocks: of rows, of a sequence's KV head
    uint32_t splits, chunk;                        // most workgroups that share a row's granules, and how many granules make one more worth it
    float c2;                                      // scale log2(e)
    uint32_t ordered;                              // whether sequences are taken by their lengths
};

constexpr float LOWEST = -3.4028234663852886e38f;  // a maximum over nothing: no finite score lies below it
// Weights are held times 2^SHIFT, relative to a maximum that moves where those of a granule come to LIMIT together: it may lie 2^11 below.  Weights down to 2^-18
// of the largest keep FP16's eleven bits, and smaller ones are off by 2^-29 of it at most.
constexpr float SHIFT = 4.0f, LIMIT = 32768.0f;
// A row's weights are 2^(c2 s + reference), and the maximum m of its scores so far decides the reference: -c2 m + SHIFT, rounded.  The product c2 s is fused with the sum, so equal scores
// have equal weights in all of a row's granules, and what the reference's rounding adds to the exponent, a quarter at most, is the same for all of them.  Where |c2 m| comes to FAR it could be
// more: the difference s - m is taken first then, which is exact where it matters.
constexpr float FAR = 4194304.0f;
__device__ __forceinline__ bool is_far(float m, float c2) { return !(fabsf(m * c2) < FAR); }           // (LOWEST is: c2 is 1e-30 or more)
__device__ __forceinline__ float reference(float m, float c2) { return __builtin_fmaf(-m, c2, SHIFT); }
// The exponent of the weight of score s under the maximum m is fma(s - less, c2, plus).
struct Exponent {
    float less, plus, c2;
    __device__ __forceinline__ Exponent(float m, float c2_) : less(is_far(m, c2_) ? m : 0.0f), plus(is_far(m, c2_) ? SHIFT : reference(m, c2_)), c2(c2_) {}
    __device__ __forceinline__ float operator()(float s) const { return __builtin_fmaf(s - less, c2, plus); }
};
// what takes sums of such weights to weights relative to 2^(c2 m) itself, but for the 2^SHIFT that all have: parts of a row meet there
__device__ __forceinline__ float own_factor(float m, float c2) { return __builtin_amdgcn_exp2f(SHIFT - Exponent(m, c2)(m)); }

// The granules that the rows r0 .. of a block see, and the parts that workgroups take of them, `chunk` each.
struct Range { uint32_t first, count, parts, chunk; };
__device__ __forceinline__ Range granules_of(const AttentionArgs &a, const Sequence &sq, uint32_t r0, uint32_t rows)
{
    const uint32_t all = (sq.n < a.max_tokens ? sq.n : a.max_tokens) * a.group;
    const uint32_t last = (r0 + rows < all ? r0 + rows : all) - 1;
    const int32_t p0 = sq.start + (int32_t)(r0 / a.group), end = sq.start + (int32_t)(last / a.group) + 1;
    const int32_t begin = a.window && (uint32_t)(p0 < 0 ? 0 : p0) >= a.window ? p0 + 1 - (int32_t)a.window : 0;
    Range g;
    g.first = (uint32_t)begin / 32u;
    g.count = end > begin ? ((uint32_t)end + 31u) / 32u - g.first : 0u;
    g.parts = 1;
    g.chunk = g.count;
    if (a.splits > 1) {
        g.parts = (g.count + a.chunk - 1) / a.chunk;
        g.parts = g.parts < 1 ? 1u : g.parts > a.splits ? a.splits : g.parts;
        g.chunk = (g.count + g.parts - 1) / g.parts;
    }
    return g;
}

// The pages of a wavefront's granules: granules `at`, `at` + step, ... of the sequence, 64 entries of the table at a time, one a lane.
template <int D> struct Walk {
    const uint8_t *base;                           // of the head in page 0
    const int32_t *row;
    uint64_t page_bytes;
    uint32_t pages, page_granules, at, step, lane;
    int32_t entry;
    __device__ __forceinline__ Walk(const CacheArgs &c, uint32_t sequence, uint32_t head, uint32_t first, uint32_t step_, uint32_t lane_)
        : base(c.cache + (uint64_t)head * c.page_granules * (34 * D)), row(c.table + sequence * c.table_stride), page_bytes((uint64_t)c.kv_heads * c.page_granules * (34 * D)),
          pages(c.pages), page_granules(c.page_granules), at(first), step(step_), lane(lane_), entry(-1) {}
    // the entries for the next 64 of the `left` granules still to come
    __device__ __forceinline__ void refill(uint32_t n, uint32_t left) { entry = lane < left ? row[(at + (n + lane) * step) / page_granules] : -1; }
    // granule n of the walk; NULL where its page is none
    __device__ __forceinline__ const uint8_t *granule(uint32_t n) const
    {
        const uint32_t page = (uint32_t)__builtin_amdgcn_readlane(entry, (int)(n & 63u)), g = (at + n * step) % page_granules;
        return page < pages ? base + page * page_bytes + g * (34 * D) : nullptr;
    }
};

// codes of bytes 0xFF in a word, as 0x80 in their bytes (exact: the lowest byte that is one is found, and those above it)
__device__ __forceinline__ uint32_t any_nan_code(uint32_t w) { return (~w - 0x01010101u) & w & 0x80808080u; }

// The conversions read the exponent field of their scale alone (all 256 fields with other bits around them: no difference), so a code needs no more than
// to be shifted there.
template <int BYTE> __device__ __forceinline__ float scale_of(uint32_t codes)
{
    return __uint_as_float(BYTE == 0 ? codes << 23 : BYTE == 1 ? codes << 15 : BYTE == 2 ? codes << 7 : codes >> 1);
}
__device__ __forceinline__ Frag16 keys_bf16(uint32_t codes, float s)
{
    Frag16 f;
    f.w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0));
    f.w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1));
    f.w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2));
    f.w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3));
    return f;
}
__device__ __forceinline__ Frag16 keys_fp16(uint32_t codes, float s)
{
    Frag16 f;
    f.w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, 0));
    f.w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, 1));
    f.w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, 2));
    f.w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, 3));
    return f;
}
// two elements of tokens 4 H .. 4 H + 3, a byte each, under those tokens' scales
template <int H> __device__ __forceinline__ void four_values(uint32_t word, const uint32_t (&scales)[2], f16x2 (&y)[8])
{
    y[4 * H] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale_of<0>(scales[H]), 0);
    y[4 * H + 1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale_of<1>(scales[H]), 1);
    y[4 * H + 2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale_of<2>(scales[H]), 2);
    y[4 * H + 3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale_of<3>(scales[H]), 3);
}

} // namespace mmaemu
