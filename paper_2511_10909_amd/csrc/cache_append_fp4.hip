// Heads of queries, keys and values on their way into attention: norm and rotation, queries in their type, keys and values into the cache.
//
//   y = x / sqrt(mean(x^2) + eps) * w;   pairs (a, b) of its first elements to (a c - b s, b c + a s);   all in binary64, rounded once to binary32
//   queries: RN_type;   keys, and values as they came: E8M0 scale per 32 elements by the rule, within 104 .. 140, elements RNE_E2M1 (saturated)
//
// Bound by memory: 2 bytes read and 2 (queries) or 17/32 (cache) written per element.  Binary64 costs nothing beside that, and codes do not depend on
// the order of a sum.
//
// A wavefront takes one head of 4 (D = 128) or 8 (D = 64) tokens whose positions share that multiple, eight consecutive elements a lane: 16 bytes
// in and out.  The cache has V's bytes of four consecutive tokens side by side: the tokens' lanes exchange them, and where all four are there, a lane
// writes four bytes at once.
#include "cache_fp4.hpp"

namespace mmaemu {

struct AppendArgs {
    CacheArgs c;
    const void *q, *k, *v, *q_weight, *k_weight;
    const float *rotation;
    void *q_out, *k_values, *v_values;
    uint64_t q_stride, k_stride, v_stride, q_out_stride;
    uint32_t heads, kv_read, vectors, blocks;      // vectors: heads of q, k and v of a token; blocks: workgroups that share a token
    uint32_t max_tokens, rotary, pairs, fit, rotation_rows;
    double eps;
};

template <int CTRL> __device__ __forceinline__ double dpp_add_all(double x)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, 0xF, 0xF, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, 0xF, 0xF, true);
    return x + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// sum over 8 or 16 consecutive lanes, in each of them
template <int LANES> __device__ __forceinline__ double sum_of_lanes(double x)
{
    x = dpp_add_all<0xB1>(x);                      // lanes 2 i and 2 i + 1
    x = dpp_add_all<0x4E>(x);                      // the other pair of four
    x = dpp_add_all<0x141>(x);                     // row_half_mirror: the other four of eight
    if (LANES == 16) x = dpp_add_all<0x140>(x);    // row_mirror: the other eight
    return x;
}

// eight values of y, of vector v of the head whose elements are x
template <int T, int TW> __device__ __forceinline__ void normed(const Raw8<T> &x, const void *weight, uint32_t v, double r, double (&y)[8])
{
    Raw8<TW> w;
    if (weight) w = load8<TW>(weight, 8 * v);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        y[i] = (double)get8<T>(x, i);
        if (weight) y[i] = y[i] * r * (double)get8<TW>(w, i);
    }
}

template <int T, int TW, int D> __global__ void __launch_bounds__(256) append_kernel(const AppendArgs a)
{
    constexpr uint32_t LANES = D / 8, TOKENS = 64 / LANES;             // of a head, of a wavefront
    const uint32_t lane = threadIdx.x & 63u, v = lane % LANES, tt = lane / LANES;
    const uint32_t vector = (blockIdx.x % a.blocks) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (vector >= a.vectors) return;
    const Sequence sq = sequence_of(a.c, blockIdx.y);
    const int32_t group = (sq.start >= 0 ? sq.start : sq.start - (int32_t)(TOKENS - 1)) / (int32_t)TOKENS + (int32_t)(blockIdx.x / a.blocks);
    const int32_t position = group * (int32_t)TOKENS + (int32_t)tt;
    const int32_t i = position - sq.start;
    const uint32_t n = sq.n < a.max_tokens ? sq.n : a.max_tokens;
    const bool here = i >= 0 && (uint32_t)i < n;
    if (!__any(here)) return;
    const uint64_t row = sq.first + (uint32_t)(here ? i : 0);

    const bool is_q = vector < a.heads, is_k = !is_q && vector < a.heads + a.kv_read;
    const uint32_t head = is_q ? vector : is_k ? vector - a.heads : vector - a.heads - a.kv_read;
    const void *from = is_q ? a.q : is_k ? a.k : a.v;
    const uint64_t stride = is_q ? a.q_stride : is_k ? a.k_stride : a.v_stride;
    Raw8<T> x = {};
    if (here) x = load8<T>(from, row * stride + head * D + 8 * v);

    float f[8];
    if (is_q || is_k) {
        const void *weight = is_q ? a.q_weight : a.k_weight;
        double r = 1.0;
        if (weight) {
            double s = 0.0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const double d = (double)get8<T>(x, e);
                s = __builtin_fma(d, d, s);
            }
            r = 1.0 / sqrt(sum_of_lanes<LANES>(s) / (double)D + a.eps);
        }
        double y[8];
        normed<T, TW>(x, weight, v, r, y);
        if (a.rotary) {
            const uint32_t half = a.rotary / 2, vectors = a.rotary / 8;            // elements; vectors that are rotated
            const bool turned = v < vectors;
            const bool held = position >= 0 && (uint32_t)position < a.rotation_rows;
            const float *table = a.rotation + (uint64_t)(uint32_t)(held ? position : 0) * a.rotary;
            if (!a.pairs) {
                const bool upper = v >= vectors / 2;
                const uint32_t other = turned ? (upper ? v - vectors / 2 : v + vectors / 2) : v;
                Raw8<T> px;
#pragma unroll
                for (int w = 0; w < 4; ++w) px.w[w] = (uint32_t)__shfl((int)x.w[w], (int)(lane - v + other));
                if (turned) {
                    double p[8];
                    normed<T, TW>(px, weight, other, r, p);
                    float c[8], s[8];
                    const uint32_t at = 8 * (upper ? other : v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) c[e] = held ? table[at + e] : __builtin_nanf(""), s[e] = held ? table[half + at + e] : 0.0f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = upper ? y[e] * (double)c[e] + p[e] * (double)s[e] : y[e] * (double)c[e] - p[e] * (double)s[e];
                }
            } else if (turned) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const double c = held ? (double)table[4 * v + e] : __builtin_nan(""), s = held ? (double)table[half + 4 * v + e] : 0.0;
                    const double y0 = y[2 * e], y1 = y[2 * e + 1];
                    y[2 * e] = y0 * c - y1 * s;
                    y[2 * e + 1] = y1 * c + y0 * s;
                }
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (float)y[e];
        if (is_q) {
            if (here) store8<T>(a.q_out, row * a.q_out_stride + head * D + 8 * v, round8<T>(f));
            return;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = get8<T>(x, e);
    }

    // codes and scale of one vector; the four lanes of a block are all here
    uint32_t amax = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t b = magnitude(f[e]);
        amax = b > amax ? b : amax;
    }
    uint32_t code = e8m0_code<2, 0x400000u>(max_of_quad(amax), a.fit), codes = 0;
    if (code != 0xFFu) {
        code = code < CACHE_SCALE_LEAST ? CACHE_SCALE_LEAST : code > CACHE_SCALE_MOST ? CACHE_SCALE_MOST : code;
        const float inverse = e8m0_inverse(code);
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = __builtin_amdgcn_fmed3f(f[e] * inverse, -6.0f, 6.0f);
        codes = pack_fp4(z);
    }
    void *values = is_k ? a.k_values : a.v_values;
    if (values && here) {
        float z[8];
        const float unit = __uint_as_float(code << 23);
        const f32x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 1),
                    p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 3);
        z[0] = p0[0]; z[1] = p0[1]; z[2] = p1[0]; z[3] = p1[1]; z[4] = p2[0]; z[5] = p2[1]; z[6] = p3[0]; z[7] = p3[1];
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = code == 0xFFu ? __builtin_nanf("") : z[e];
        store8<T>(values, row * ((uint64_t)a.c.kv_heads * D) + head * D + 8 * v, round8<T>(z));
    }

    // the wavefront's granule; the positions of its tokens share it, and where one of them is the sequence's, it is in the table's row
    const uint32_t t = (uint32_t)position % 32u, w = t / 8, half = t / 4 % 2, in_four = t % 4;
    if (group < 0) return;
    const uint32_t granule = (uint32_t)group * TOKENS / 32u;
    uint8_t *const g = granule_at<D>(a.c, a.c.table[blockIdx.y * a.c.table_stride + granule / a.c.page_granules], head, granule % a.c.page_granules);
    if (!g) return;
    if (is_k) {
        if (!here) return;
        const uint32_t at = D == 128 ? half * 1024 + v / 4 * 256 + (4 * w + in_four) * 16 + v % 4 * 4 : v / 2 * 256 + (4 * w + in_four) * 16 + half * 8 + v % 2 * 4;
        *reinterpret_cast<uint32_t *>(g + at) = codes;
        if (v % 4 == 0) g[32 * D + (16 * (v / 4) + 4 * w + in_four) * 2 + half] = (uint8_t)code;
        return;
    }
    // V: the byte of element pair j (of four) of vector `vec`, token 0 of eight
    const auto pair_at = [&](uint32_t vec, uint32_t j) {
        return 16u * D + (D == 128 ? j / 2 * 1024 + w * 256 + vec * 16 + j % 2 * 8 : w * 256 + (2 * vec + j / 2) * 16 + j % 2 * 8);
    };
    // four tokens side by side, the first of them lane group `base`: this lane takes pair j of its vector
    const uint32_t base = TOKENS == 4 ? 0u : 4 * (tt & 1u), j = TOKENS == 4 ? tt : tt / 2;
    const uint64_t present = __ballot(here);
    const auto all_four = [&](uint32_t first) {
        bool all = true;
#pragma unroll
        for (uint32_t s = 0; s < 4; ++s) all = all && (present >> ((first + s) * LANES) & 1u);
        return all;
    };
    uint32_t four = 0;
#pragma unroll
    for (uint32_t s = 0; s < 4; ++s) four |= ((uint32_t)__shfl((int)codes, (int)((base + s) * LANES + v)) >> (8 * j) & 0xFFu) << (8 * s);
    if (all_four(base)) *reinterpret_cast<uint32_t *>(g + pair_at(v, j) + (TOKENS == 4 ? 4 * half : base)) = four;
    if (!here) return;
    // a token whose four are not all there writes its own bytes
    if (!all_four(tt / 4 * 4)) {
#pragma unroll
        for (uint32_t p = 0; p < 4; ++p) g[pair_at(v, p) + t % 8] = (uint8_t)(codes >> (8 * p));
    }
    if (v % 4 == 0) g[33 * D + (w * (D / 32) + v / 4) * 8 + t % 8] = (uint8_t)code;
}

mmaemu_status launch_cache_append(const mmaemu_cache_append_fp4_args &a, const CacheArgs &c, hipStream_t s)
{
    const uint32_t kv_read = a.k ? c.kv_heads : 0, vectors = a.heads + 2 * kv_read, per = a.dim == 128 ? 4 : 8;
    const AppendArgs p = {c, a.q, a.k, a.v, a.q_weight, a.k_weight, a.rotation, a.q_out, a.k_values, a.v_values, a.q_stride, a.k_stride, a.v_stride, a.q_out_stride,
                          a.heads, kv_read, vectors, (vectors + 3) / 4, a.max_tokens, a.rotary_dim, a.rotation_style == MMAEMU_ROTATE_PAIRS,
                          a.scale_rule == MMAEMU_SCALE_RULE_FIT, (uint32_t)(a.rotation_rows < 0x7FFFFFFF ? a.rotation_rows : 0x7FFFFFFF), a.eps};
    // groups of `per` positions that max_tokens consecutive ones may touch
    const dim3 grid(((a.max_tokens + per - 2) / per + 1) * p.blocks, a.sequences);
    const bool wide = a.weight_type == MMAEMU_FP32;
#define MMAEMU_APPEND(T, TW)                                                                                          \
    do {                                                                                                              \
        if (a.dim == 128) hipLaunchKernelGGL((append_kernel<T, TW, 128>), grid, dim3(256), 0, s, p);                  \
        else hipLaunchKernelGGL((append_kernel<T, TW, 64>), grid, dim3(256), 0, s, p);                                \
    } while (0)
    if (a.type == MMAEMU_BF16) {
        if (wide) MMAEMU_APPEND(MMAEMU_BF16, MMAEMU_FP32);
        else MMAEMU_APPEND(MMAEMU_BF16, MMAEMU_BF16);
    } else {
        if (wide) MMAEMU_APPEND(MMAEMU_FP16, MMAEMU_FP32);
        else MMAEMU_APPEND(MMAEMU_FP16, MMAEMU_FP16);
    }
#undef MMAEMU_APPEND
    MMAEMU_HIP(hipGetLastError());
    return MMAEMU_OK;
}

} // namespace mmaemu
