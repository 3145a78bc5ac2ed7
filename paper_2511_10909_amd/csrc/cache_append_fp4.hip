// Heads of queries, keys and values on their way into attention: norm and rotation, queries in their type, keys and values into the cache.
//
//   y = x / sqrt(mean(x^2) + eps) * w;   pairs (a, b) of its first elements to (a c - b s, b c + a s);   all in binary64, rounded once to binary32
//   queries: RN_type;   keys, and values as they came: E8M0 scale per 32 elements by the rule, within 104 .. 140, elements RNE_E2M1 (saturated)
//
// Bound by memory: 2 bytes read and 2 (queries) or 17/32 (cache) written per element.  Binary64 costs little beside that, and codes do not depend on
// the order of a sum.  8192 tokens of 32 + 2 x 8 heads of 128 in BF16: 52 us, 4.1 TB/s (a copy reaches 5.15), vector instructions in 59 % of the cycles.
//
// A lane holds eight consecutive elements of a head: 16 bytes in and out.  Where several tokens of a sequence come, a wavefront takes 4 (D = 128) or 8
// (D = 64) tokens whose positions share that multiple, and some heads one after another: weights times cosines and sines, the same for all of them,
// are made once, so that a rotated element is (r x) wc + (r x') ws.  The cache has V's bytes of four consecutive tokens side by side: the tokens' lanes
// exchange them, and where all four are there, a lane writes four bytes at once.  Where one or two tokens come, a wavefront takes 4 or 8 heads of one.
#include "cache_fp4.hpp"
#include <type_traits>

namespace mmaemu {

struct AppendArgs {
    CacheArgs c;
    const void *q, *k, *v, *q_weight, *k_weight;
    const float *rotation;
    void *q_out, *k_values, *v_values;
    uint64_t q_stride, k_stride, v_stride, q_out_stride;
    uint32_t heads, kv_read, per;                  // per: heads that a wavefront takes one after another
    uint32_t units, q_units, kv_units;             // wavefronts that share a token or group of tokens, for queries, and for keys or values
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

// 1 / sqrt(x) within two units in the last place: the instruction's approximation and two steps of Newton's method (zero and infinity as it has them)
__device__ __forceinline__ double inverse_sqrt(double x)
{
    const double r0 = __builtin_amdgcn_rsq(x);
    const double e0 = __builtin_fma(-x * r0, r0, 1.0), r1 = __builtin_fma(r0 * 0.5, e0, r0);
    const double e1 = __builtin_fma(-x * r1, r1, 1.0), r2 = __builtin_fma(r1 * 0.5, e1, r1);
    return x == 0.0 || x == __builtin_inf() ? r0 : r2;
}

// What a lane multiplies its elements (x) and their partners (x') by: weights and the rotation's cosines and signed sines.  `at`: the lane's
// first cosine, NULL where it turns nothing (lost: where the table has none for the position); other: the vector that has the partners.
template <int TW> __device__ __forceinline__ void factors(const AppendArgs &a, const void *weight, const float *at, bool lost, bool upper, uint32_t v, uint32_t other,
                                                          double (&wc)[8], double (&ws)[8])
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {                  // four elements at a time
        float c[4], s[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] = lost ? __builtin_nanf("") : 1.0f, s[e] = 0.0f;
        if (at && a.pairs) {
            const Words2<4> x = reinterpret_cast<const Words2<4> *>(at)[h], y = reinterpret_cast<const Words2<4> *>(at + a.rotary / 2)[h];
#pragma unroll
            for (int e = 0; e < 4; ++e) c[e] = word_float(x.w[e / 2]), s[e] = word_float(y.w[e / 2] ^ (e % 2 ? 0u : 0x80000000u));
        } else if (at) {
            const Words4<4> x = reinterpret_cast<const Words4<4> *>(at)[h], y = reinterpret_cast<const Words4<4> *>(at + a.rotary / 2)[h];
#pragma unroll
            for (int e = 0; e < 4; ++e) c[e] = word_float(x.w[e]), s[e] = word_float(y.w[e] ^ (upper ? 0u : 0x80000000u));
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) wc[4 * h + e] = (double)c[e], ws[4 * h + e] = (double)s[e];
    }
    if (weight) {
        const Raw8<TW> w = load8<TW>(weight, 8 * v), p = load8<TW>(weight, 8 * other);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            wc[e] *= (double)get8<TW>(w, e);
            ws[e] *= (double)(a.pairs ? get8<TW>(w, e ^ 1) : get8<TW>(p, e));
        }
    }
}

enum { KIND_Q = 0, KIND_K = 1, KIND_V = 2 };

// HEADS: the lanes' groups are heads of one token, else tokens of one head.
template <int T, int TW, int D, bool HEADS> __global__ void __launch_bounds__(256, 4) append_kernel(const AppendArgs a)
{
    constexpr uint32_t LANES = D / 8, GROUPS = 64 / LANES;             // of a head, of a wavefront
    const uint32_t lane = threadIdx.x & 63u, v = lane % LANES, tt = lane / LANES;
    const uint32_t wave = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), share = wave % a.units, nth = wave / a.units;
    const Sequence sq = sequence_of(a.c, blockIdx.y);
    const uint32_t n = sq.n < a.max_tokens ? sq.n : a.max_tokens;
    // the lane's token
    int32_t first = 0;
    bool here;
    int32_t i;
    if (HEADS) {
        i = (int32_t)nth;
        here = nth < n;
    } else {
        first = ((sq.start >= 0 ? sq.start : sq.start - (int32_t)(GROUPS - 1)) / (int32_t)GROUPS + (int32_t)nth) * (int32_t)GROUPS;
        i = first + (int32_t)tt - sq.start;
        here = i >= 0 && (uint32_t)i < n;
    }
    if (!__any(here)) return;
    const int32_t position = sq.start + i;
    const uint64_t row = sq.first + (uint32_t)(here ? i : 0);

    // the granule; the positions of a wavefront's tokens share it, and where one of them is the sequence's, it is in the table's row
    const uint32_t place = HEADS ? (uint32_t)position : (uint32_t)first;
    const bool in_cache = (int32_t)place >= 0;
    int32_t page = -1;
    if (in_cache) page = a.c.table[blockIdx.y * a.c.table_stride + place / 32u / a.c.page_granules];
    const uint32_t t = (uint32_t)position % 32u, w = t / 8, half = t / 4 % 2, in_four = t % 4;

    // cosines and signed sines of the lane's elements, and the lane that has their partners
    const uint32_t turned = a.rotary / 8;          // vectors of a head that are rotated
    const bool turns = v < turned, upper = v >= turned / 2;
    const uint32_t other = turns && !a.pairs ? (upper ? v - turned / 2 : v + turned / 2) : v;
    const bool held = position >= 0 && (uint32_t)position < a.rotation_rows;
    const float *angles = nullptr;
    if (turns && held) angles = a.rotation + (uint64_t)(uint32_t)position * a.rotary + (a.pairs ? 4 * v : 8 * (upper ? other : v));

    // `per` heads of one kind, one after another (HEADS: GROUPS heads at once)
    const auto heads_of_kind = [&](auto which, uint32_t nth_share) __attribute__((always_inline)) {
        constexpr int kind = decltype(which)::value;
        const uint32_t count = kind == KIND_Q ? a.heads : a.kv_read;
        const uint32_t x0 = HEADS ? nth_share : nth_share * a.per, x1 = HEADS ? x0 + 1 : x0 + a.per < count ? x0 + a.per : count;
        const void *const from = kind == KIND_Q ? a.q : kind == KIND_K ? a.k : a.v;
        const uint64_t in = row * (kind == KIND_Q ? a.q_stride : kind == KIND_K ? a.k_stride : a.v_stride) + 8 * v;
        const auto head_of = [&](uint32_t x) { return HEADS ? x * GROUPS + tt : x; };
        const auto load = [&](uint32_t x) {
            Raw8<T> r = {};
            if (here && (!HEADS || head_of(x) < count)) r = load8<T>(from, in + head_of(x) * D);
            return r;
        };
        const void *const weight = kind == KIND_Q ? a.q_weight : kind == KIND_K ? a.k_weight : nullptr;
        double wc[8], ws[8];
        Raw8<T> next = load(x0);
        if (kind != KIND_V) factors<TW>(a, weight, angles, turns && !held, upper, v, other, wc, ws);
        for (uint32_t vector = x0; vector < x1; ++vector) {
            const Raw8<T> x = next;
            if (!HEADS && vector + 1 < x1) next = load(vector + 1);
            const uint32_t head = head_of(vector);
            const bool mine = here && (!HEADS || head < count);
            float f[8];
            if constexpr (kind != KIND_V) {
                double r = 1.0;
                if (weight) {
                    double sum = 0.0;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const double d = (double)get8<T>(x, e);
                        sum = __builtin_fma(d, d, sum);
                    }
                    r = inverse_sqrt(__builtin_fma(sum_of_lanes<LANES>(sum), 1.0 / D, a.eps));
                }
                if (a.rotary) {
                    Raw8<T> px;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        px.w[e] = a.pairs ? x.w[e] >> 16 | x.w[e] << 16 : (uint32_t)__shfl((int)x.w[e], (int)(lane - v + other));
                        px.w[e] = turns ? px.w[e] : 0u;                // (an infinity that is not turned stays one)
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] = (float)__builtin_fma((double)get8<T>(x, e) * r, wc[e], (double)get8<T>(px, e) * r * ws[e]);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] = (float)((double)get8<T>(x, e) * r * wc[e]);
                }
                if constexpr (kind == KIND_Q) {
                    if (mine) store8<T>(a.q_out, row * a.q_out_stride + head * D + 8 * v, round8<T>(f));
                    continue;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = get8<T>(x, e);
            }
            if constexpr (kind != KIND_Q) {
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
                void *values = kind == KIND_K ? a.k_values : a.v_values;
                if (values && mine) {
                    float z[8];
                    const float unit = __uint_as_float(code << 23);
                    const f32x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 1),
                                p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, unit, 3);
                    z[0] = p0[0]; z[1] = p0[1]; z[2] = p1[0]; z[3] = p1[1]; z[4] = p2[0]; z[5] = p2[1]; z[6] = p3[0]; z[7] = p3[1];
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[e] = code == 0xFFu ? __builtin_nanf("") : z[e];
                    store8<T>(values, row * ((uint64_t)a.c.kv_heads * D) + head * D + 8 * v, round8<T>(z));
                }

                if (!in_cache) continue;
                uint8_t *const g = granule_at<D>(a.c, page, head, place / 32u % a.c.page_granules);
                if (!g) continue;
                if constexpr (kind == KIND_K) {
                    if (!mine) continue;
                    const uint32_t at = D == 128 ? half * 1024 + v / 4 * 256 + (4 * w + in_four) * 16 + v % 4 * 4 : v / 2 * 256 + (4 * w + in_four) * 16 + half * 8 + v % 2 * 4;
                    *reinterpret_cast<uint32_t *>(g + at) = codes;
                    if (v % 4 == 0) g[32 * D + (16 * (v / 4) + 4 * w + in_four) * 2 + half] = (uint8_t)code;
                    continue;
                }
                // V: the byte of element pair j (of four) of this lane's vector, token 0 of eight
                const auto pair_at = [&](uint32_t j) {
                    return 16u * D + (D == 128 ? j / 2 * 1024 + w * 256 + v * 16 + j % 2 * 8 : w * 256 + (2 * v + j / 2) * 16 + j % 2 * 8);
                };
                bool alone = true;
                if (!HEADS) {
                    // four tokens side by side, the first of them lane group `base`: this lane takes pair j of its vector
                    const uint32_t base = GROUPS == 4 ? 0u : 4 * (tt & 1u), j = GROUPS == 4 ? tt : tt / 2;
                    const uint64_t present = __ballot(here);
                    const auto all_four = [&](uint32_t group) {
                        bool all = true;
#pragma unroll
                        for (uint32_t e = 0; e < 4; ++e) all = all && (present >> ((group + e) * LANES) & 1u);
                        return all;
                    };
                    uint32_t four = 0;
#pragma unroll
                    for (uint32_t e = 0; e < 4; ++e) four |= ((uint32_t)__shfl((int)codes, (int)((base + e) * LANES + v)) >> (8 * j) & 0xFFu) << (8 * e);
                    if (all_four(base)) *reinterpret_cast<uint32_t *>(g + pair_at(j) + (GROUPS == 4 ? 4 * half : base)) = four;
                    alone = !all_four(tt / 4 * 4);
                }
                if (!mine) continue;
                if (alone) {                               // a token whose four are not all there writes its own bytes
#pragma unroll
                    for (uint32_t p = 0; p < 4; ++p) g[pair_at(p) + t % 8] = (uint8_t)(codes >> (8 * p));
                }
                if (v % 4 == 0) g[33 * D + (w * (D / 32) + v / 4) * 8 + t % 8] = (uint8_t)code;
            }
        }
    };

    // the wavefront's share of a token: some heads of q, of k or of v
    if (share < a.q_units) heads_of_kind(std::integral_constant<int, KIND_Q>(), share);
    else if (share < a.q_units + a.kv_units) heads_of_kind(std::integral_constant<int, KIND_K>(), share - a.q_units);
    else heads_of_kind(std::integral_constant<int, KIND_V>(), share - a.q_units - a.kv_units);
}

mmaemu_status launch_cache_append(const mmaemu_cache_append_fp4_args &a, const CacheArgs &c, hipStream_t s)
{
    const uint32_t kv_read = a.k ? c.kv_heads : 0, groups = a.dim == 128 ? 4 : 8;
    const bool by_heads = a.max_tokens <= 2, wide = a.weight_type == MMAEMU_FP32;
    // groups of positions that max_tokens consecutive ones may touch
    const uint32_t parts = by_heads ? a.max_tokens : (a.max_tokens + groups - 2) / groups + 1;
    // Heads of a wavefront, us (8192 tokens of 32 + 2 x 8 heads of 128; five chunks of up to 1499 tokens, 12 + 2 x 4 of 64): one 11.6 for the latter, two 66 and 10.5,
    // four 55 and 11.5, eight 52 and 13, twelve 53 and 12.6
    const uint64_t all = (uint64_t)parts * (a.heads + 2 * kv_read) * a.sequences;
    const uint32_t per = by_heads ? 1 : all >= 65536 ? 8 : all >= 8192 ? 2 : 1, at_once = by_heads ? groups : per;
    const uint32_t q_units = (a.heads + at_once - 1) / at_once, kv_units = (kv_read + at_once - 1) / at_once, units = q_units + 2 * kv_units;
    const AppendArgs p = {c, a.q, a.k, a.v, a.q_weight, a.k_weight, a.rotation, a.q_out, a.k_values, a.v_values, a.q_stride, a.k_stride, a.v_stride, a.q_out_stride,
                          a.heads, kv_read, per, units, q_units, kv_units, a.max_tokens, a.rotary_dim, a.rotation_style == MMAEMU_ROTATE_PAIRS,
                          a.scale_rule == MMAEMU_SCALE_RULE_FIT, (uint32_t)(a.rotation_rows < 0x7FFFFFFF ? a.rotation_rows : 0x7FFFFFFF), a.eps};
    const dim3 grid((parts * units + 3) / 4, a.sequences);
#define MMAEMU_APPEND(T, TW, D)                                                                                       \
    do {                                                                                                              \
        if (by_heads) hipLaunchKernelGGL((append_kernel<T, TW, D, true>), grid, dim3(256), 0, s, p);                  \
        else hipLaunchKernelGGL((append_kernel<T, TW, D, false>), grid, dim3(256), 0, s, p);                          \
    } while (0)
#define MMAEMU_APPEND_TYPED(T, TW)                  \
    do {                                            \
        if (a.dim == 128) MMAEMU_APPEND(T, TW, 128); \
        else MMAEMU_APPEND(T, TW, 64);              \
    } while (0)
    if (a.type == MMAEMU_BF16) {
        if (wide) MMAEMU_APPEND_TYPED(MMAEMU_BF16, MMAEMU_FP32);
        else MMAEMU_APPEND_TYPED(MMAEMU_BF16, MMAEMU_BF16);
    } else {
        if (wide) MMAEMU_APPEND_TYPED(MMAEMU_FP16, MMAEMU_FP32);
        else MMAEMU_APPEND_TYPED(MMAEMU_FP16, MMAEMU_FP16);
    }
#undef MMAEMU_APPEND_TYPED
#undef MMAEMU_APPEND
    MMAEMU_HIP(hipGetLastError());
    return MMAEMU_OK;
}

} // namespace mmaemu
