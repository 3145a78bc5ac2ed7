// Attention over the cache in 4 bits: out = softmax(scale q K^T) V over the tokens that a row sees, from one token to prompts.
//
// The rows of a KV head are its group's query heads of all the call's tokens of a sequence, r = token * group + head: they share K and V.  One pass
// over the tokens with a running maximum m and sum l per row, c = scale log2(e):
//   s = q.k;  m' = max(m, max s);  p = 2^(c (s - m'));  l = l 2^(c (m - m')) + sum p;  O = O 2^(c (m - m')) + p V;  out = O / l
// Both products are 16 x 16 x 32 instructions on operands that lie in the cache as the lanes take them (cache_fp4.hpp), brought to 16 bits, which is
// exact: K to the queries' type, V to FP16.  The scores' registers are the second product's operand as they are, rounded to FP16.
//
// Few rows are bound by memory: 64 sequences of up to 16384 tokens, 64 heads over 8 of 128, 148 us, 4.9 TB/s.  Prompts are bound by the SIMDs' issue port, which matrix
// instructions hold for ten cycles, exponentials for eight and other vector instructions for four: 8192 tokens x 32 heads 540 us, 1.0 PFLOP/s of the products that are needed.
#include "attention_fp4.hpp"

#include <cstdio>

namespace mmaemu {

__device__ __forceinline__ float other_rows_max(float x)               // over lanes l, l + 16, l + 32, l + 48
{
    const uint32_t b = __float_as_uint(x);
    const auto p = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    const float y = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    const uint32_t c = __float_as_uint(y);
    const auto q = __builtin_amdgcn_permlane16_swap(c, c, false, false);
    return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}

// a granule as a lane holds it: keys with the scales of both halves, values with the scales of eight tokens
template <int D> struct Keys { u32x4 k[D / 64]; uint32_t scales; };
template <int D> struct Values { u32x4 v[D / 64]; uint32_t scales[2]; };
// A lane's places in a granule.  Their values are hidden, so that a load adds them to the granule's uniform address by itself.
template <int D> struct Offsets {
    uint32_t codes, key_scales, value_scales;
    __device__ __forceinline__ explicit Offsets(uint32_t lane)
    {
        constexpr uint32_t B = D / 32;
        codes = 16 * lane;
        key_scales = 32 * D + ((lane >> 4) * B / 4 * 16 + (lane & 15u)) * 2;
        value_scales = 33 * D + ((lane >> 4) * B + (lane & 15u) * B / 16) * 8;
        asm volatile("" : "+v"(codes), "+v"(key_scales), "+v"(value_scales));
    }
};
template <int D> __device__ __forceinline__ void load_keys(Keys<D> &x, const uint8_t *at, const Offsets<D> &off)
{
#pragma unroll
    for (int i = 0; i < D / 64; ++i) x.k[i] = *reinterpret_cast<const u32x4 *>(at + 1024 * i + off.codes);
    x.scales = *reinterpret_cast<const uint16_t *>(at + off.key_scales);
}
template <int D> __device__ __forceinline__ void load_values(Values<D> &x, const uint8_t *at, const Offsets<D> &off)
{
#pragma unroll
    for (int i = 0; i < D / 64; ++i) x.v[i] = *reinterpret_cast<const u32x4 *>(at + 16 * D + 1024 * i + off.codes);
    const Words2<8> w = *reinterpret_cast<const Words2<8> *>(at + off.value_scales);
    x.scales[0] = w.w[0];
    x.scales[1] = w.w[1];
}

// the 16-bit K operand of half A, elements 8 j .. 8 j + 7 of the lane's D / 4
template <int T, int D, int A> __device__ __forceinline__ Frag16 k_operand(const Keys<D> &x, int j)
{
    const uint32_t word = D == 128 ? x.k[D == 128 ? A : 0][j] : x.k[0][2 * A + j];
    return T == MMAEMU_BF16 ? keys_bf16(word, scale_of<A>(x.scales)) : keys_fp16(word, scale_of<A>(x.scales));
}

// The sequence of rank k by length, the longest first (up to 64 of them; equal ones in order).  Workgroups start in the order of their indexes, and where few of them fill
// the chip, the last to start should have the least to do: six chunks of 391 to 1030 tokens over 2159 to 6007 take 323 us in
// that order, 406 in the call's.  (Prompts by themselves are not put in order: their own workgroups see from nothing to all; four of up to 4000 tokens 390 us, 371 without.)
__device__ __forceinline__ uint32_t by_length(const CacheArgs &c, uint32_t k)
{
    const uint32_t lane = threadIdx.x & 63u;
    const int32_t length = lane < c.sequences ? c.lengths[lane] : 0;
    uint32_t rank = 0;
    for (uint32_t j = 0; j < c.sequences; ++j) {
        const int32_t other = __builtin_amdgcn_readlane(length, (int)j);
        rank += other > length || (other == length && j < lane);
    }
    return (uint32_t)__builtin_ctzll(__ballot(lane < c.sequences && rank == k));
}

// Rows of NR x 16 x ROW_WAVES, tokens split over the other wavefronts.  Where the tiles of rows are many, the queries wait in LDS.  As many wavefronts a SIMD as registers
// allow without scratch memory in the loop: two tiles of heads of 128 at three 134 us, at two 105 (3000 tokens x 32 heads); three tiles of heads of 64 at two 386 us,
// at three 340 (8192 tokens x 32 heads).
template <int T, int D, int NR, int ROW_WAVES, int WAVES> __global__ void __launch_bounds__(64 * WAVES, NR == 1 || (NR == 2 && D == 64) ? 4 : D == 64 ? 3 : 2) attention_kernel(const AttentionArgs a)
{
    constexpr uint32_t TOKEN_WAVES = WAVES / ROW_WAVES, J = D / 32, DT = D / 16;
    constexpr uint32_t ROWS = 16 * NR * ROW_WAVES;
    constexpr bool Q_LDS = NR >= 4;
    __shared__ __attribute__((aligned(16))) float lds[TOKEN_WAVES > 1 ? TOKEN_WAVES * 16 * (D + 4) : 1];
    __shared__ f32x2 lds_stat[TOKEN_WAVES > 1 ? TOKEN_WAVES * 16 * NR : 1];
    __shared__ u32x4 lds_q[Q_LDS ? ROW_WAVES * NR * J * 64 : 1];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, l = lane & 15u;
    const uint32_t head = blockIdx.x % a.c.kv_heads, block = a.blocks - 1 - blockIdx.x / a.c.kv_heads;        // the longest rows first
    const uint32_t split = blockIdx.y, s = ROW_WAVES > 1 && a.ordered ? by_length(a.c, blockIdx.z) : blockIdx.z;
    const Sequence sq = sequence_of(a.c, s);
    const uint32_t rows = (sq.n < a.max_tokens ? sq.n : a.max_tokens) * a.group;
    if (block * ROWS >= rows) return;
    const Range range = granules_of(a, sq, block * ROWS, ROWS);
    if (split >= range.parts) return;
    const uint32_t begin = split * range.chunk;
    uint32_t count = range.count > begin ? (range.count - begin < range.chunk ? range.count - begin : range.chunk) : 0u;
    const bool direct = range.parts == 1;
    const uint32_t r0 = block * ROWS + (ROW_WAVES > 1 ? wave * 16 * NR : 0);
    // positions of the wavefront's first and last rows; its granules
    const uint32_t r_last = (r0 + 16 * NR < rows ? r0 + 16 * NR : rows) - 1;
    const int32_t pos_first = sq.start + (int32_t)(r0 / a.group), pos_last = r0 < rows ? sq.start + (int32_t)(r_last / a.group) : -1;
    const uint32_t ends = pos_last < 0 ? 0u : (uint32_t)pos_last / 32u + 1, from = range.first + begin;
    if (ROW_WAVES > 1) count = ends > from ? (ends - from < count ? ends - from : count) : 0u;
    const uint32_t skip = ROW_WAVES > 1 ? 0 : wave, mine = count > skip ? (count - skip + TOKEN_WAVES - 1) / TOKEN_WAVES : 0u;
    Walk<D> walk(a.c, s, head, from + skip, TOKEN_WAVES, lane);
    walk.refill(0, mine);

    // this lane's rows: query operands, and positions (rows that are not there: the last one again)
    Frag16 q[Q_LDS ? 1 : NR][J];
    u32x4 *const wave_q = lds_q + (ROW_WAVES > 1 ? wave * (NR * J * 64) : 0) + lane;
    uint32_t apart = 0;                            // bytes: how far a tile's row lies behind the wavefront's first position (less than 64 tokens)
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const uint32_t r = r0 + 16 * i + l < rows ? r0 + 16 * i + l : rows - 1, token = r / a.group, h = r % a.group;
        apart |= (token - r0 / a.group & 0xFFu) << (8 * i);
        if (Q_LDS && ROW_WAVES == 1 && (uint32_t)i % WAVES != wave) continue;      // (the same for all wavefronts: they share them)
        const uint16_t *at = (const uint16_t *)a.q + (uint64_t)(sq.first + token) * a.q_stride + (uint64_t)(head * a.group + h) * D + g * (D / 4);
#pragma unroll
        for (uint32_t j = 0; j < J; ++j) {
            const u32x4 w = *reinterpret_cast<const u32x4 *>(at + 8 * j);
            if constexpr (Q_LDS) wave_q[(i * J + j) * 64] = w;
            else q[i][j].w = w;
        }
    }

    if (Q_LDS && ROW_WAVES == 1) __syncthreads();

    const Frag16 ones = {{0x3C003C00u, 0x3C003C00u, 0x3C003C00u, 0x3C003C00u}};
    float m[NR];
    f32x4 acc[NR][DT];
    float sum[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        m[i] = LOWEST;
        sum[i] = 0.0f;
#pragma unroll
        for (uint32_t d = 0; d < DT; ++d) acc[i][d] = f32x4{0, 0, 0, 0};
    }

    // The next granule's keys are read once this one's are used, its values once this one's are: they are on their way during the other's products.
    // (Where a page is none, and past the end, the first granule of the memory is read: a load that always happens costs no branch.)
    bool there = false;
    float c2 = a.c2;                               // NaN once a maximum is far, so that all weights are made again (a flag beside it: 559 us, 541 without, 8192 tokens x 32 heads)
    const uint8_t *at = walk.base;
    const auto advance = [&](uint32_t n) MMAEMU_INLINE {
        if ((n & 63u) == 0 && n && n < mine) walk.refill(n, mine - n);
        const uint8_t *const next = n < mine ? walk.granule(n) : nullptr;
        there = next != nullptr;
        at = there ? next : walk.base;
    };
    const Offsets<D> off(lane);
    Keys<D> xk;
    Values<D> xv;
    advance(0);
    load_keys<D>(xk, at, off);
    load_values<D>(xv, at, off);
    for (uint32_t n = 0; n < mine; ++n) {
        const bool now = there;
        advance(n + 1);
        if (!now) {
            load_keys<D>(xk, at, off);
            load_values<D>(xv, at, off);
            continue;
        }
        const int32_t t0 = (int32_t)(32 * (from + skip + n * TOKEN_WAVES));
        // whether all rows see all of the granule
        const bool whole = t0 + 31 <= pos_first && (!a.window || (uint32_t)(pos_last - t0) < a.window);
        // the lane's first token and its rows' distances, for branches that few granules take: their values are hidden, or what is made of them would be made for all
        struct Mask { int32_t t; uint32_t apart; };
        const auto mask = [&]() {
            Mask x = {t0 + 8 * (int32_t)g, apart};
            asm volatile("" : "+v"(x.t), "+v"(x.apart));
            return x;
        };
        const auto sees = [&](const Mask &x, int e, int i) {
            const int32_t behind = pos_first + (int32_t)(x.apart >> (8 * i) & 0xFFu) - (x.t + e);
            return behind >= 0 && (!a.window || (uint32_t)behind < a.window);
        };
        if (!whole) {
            // tokens that no row sees may hold anything: their V scales become the least
            const int32_t t = mask().t;
            const int32_t low = a.window && (uint32_t)(pos_first < 0 ? 0 : pos_first) >= a.window ? pos_first + 1 - (int32_t)a.window : 0;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (t + e > pos_last || t + e < low) xv.scales[e / 4] &= ~(0xFFu << (8 * (e % 4)));
        }
        // scores: half h, register e is token 8 g + 4 h + e
        f32x4 sc[NR][2];
#pragma unroll
        for (int i = 0; i < NR; ++i) sc[i][0] = sc[i][1] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (uint32_t j = 0; j < J; ++j) {
            const Frag16 k0 = k_operand<T, D, 0>(xk, (int)j), k1 = k_operand<T, D, 1>(xk, (int)j);
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                Frag16 qi;
                if constexpr (Q_LDS) qi.w = wave_q[(i * J + j) * 64];
                else qi = q[i][j];
                sc[i][0] = T == MMAEMU_BF16 ? mfma_bf16(k0, qi, sc[i][0]) : mfma_fp16(k0, qi, sc[i][0]);
                sc[i][1] = T == MMAEMU_BF16 ? mfma_bf16(k1, qi, sc[i][1]) : mfma_fp16(k1, qi, sc[i][1]);
            }
        }
        load_keys<D>(xk, at, off);
        if (!whole) {
            const Mask x = mask();
#pragma unroll
            for (int i = 0; i < NR; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) sc[i][e / 4][e % 4] = sees(x, e, i) ? sc[i][e / 4][e % 4] : -__builtin_inff();
        }
        // Weights against the maximum as it was, and their sums over the granule, which the matrix instruction makes as well.  Where a tile's sum comes to LIMIT (or is
        // NaN, or a weight has left FP16), its maxima move and its weights are made again.
        Frag16 p[NR];
        float add[NR];
        f32x4 total[NR];
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const float off = reference(m[i], a.c2);
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const f32x2 y = {__builtin_amdgcn_exp2f(__builtin_fmaf(sc[i][e / 4][e % 4], c2, off)),
                                 __builtin_amdgcn_exp2f(__builtin_fmaf(sc[i][e / 4][e % 4 + 1], c2, off))};
                p[i].w[e / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(y, f16x2));
            }
            total[i] = mfma_fp16(ones, p[i], f32x4{0, 0, 0, 0});
        }
        bool over = false;
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            add[i] = total[i][0];
            over = over || !(add[i] < LIMIT);
        }
        if (__any(over)) {
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                if (!__any(!(add[i] < LIMIT))) continue;
                float top = fmaxf(fmaxf(sc[i][0][0], sc[i][0][1]), fmaxf(sc[i][0][2], sc[i][0][3]));
                top = fmaxf(top, fmaxf(fmaxf(sc[i][1][0], sc[i][1][1]), fmaxf(sc[i][1][2], sc[i][1][3])));
                top = fmaxf(m[i], other_rows_max(top));
                // from one reference to the other: what both make of the new maximum's own weight
                const Exponent before(m[i], a.c2), now(top, a.c2);
                const float factor = __builtin_amdgcn_exp2f(now(top) - before(top));
                m[i] = top;
                sum[i] *= factor;
#pragma unroll
                for (uint32_t d = 0; d < DT; ++d) acc[i][d] *= factor;
                if (__any(is_far(top, a.c2) && top != LOWEST)) c2 = __builtin_nanf("");
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const f32x2 y = {__builtin_amdgcn_exp2f(now(sc[i][e / 4][e % 4])), __builtin_amdgcn_exp2f(now(sc[i][e / 4][e % 4 + 1]))};
                    p[i].w[e / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(y, f16x2));
                }
                add[i] = mfma_fp16(ones, p[i], f32x4{0, 0, 0, 0})[0];
            }
        }
#pragma unroll
        for (int i = 0; i < NR; ++i) sum[i] += add[i];
        // NaN blocks among the values: they are taken as zeros, and make NaN the outputs of the rows that see them
        if (__any(any_nan_code(xv.scales[0]) | any_nan_code(xv.scales[1]))) {
            const Mask x = mask();
            f16x8 bad;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool nan = (xv.scales[e / 4] >> (8 * (e % 4)) & 0xFFu) == 0xFFu;
                bad[e] = nan ? (_Float16)1.0f : (_Float16)0.0f;
                if (nan) xv.scales[e / 4] &= ~(0xFFu << (8 * (e % 4)));
            }
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                f16x8 seen;
#pragma unroll
                for (int e = 0; e < 8; ++e) seen[e] = sees(x, e, i) ? (_Float16)1.0f : (_Float16)0.0f;
                const f32x4 hit = __builtin_amdgcn_mfma_f32_16x16x32_f16(bad, seen, f32x4{0, 0, 0, 0}, 0, 0, 0);
#pragma unroll
                for (uint32_t d = 0; d < DT; ++d)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][d][e] = hit[e] > 0.0f ? __builtin_nanf("") : acc[i][d][e];
            }
        }
        // values: word pairs of two elements 2 c, 2 c + 1 and eight tokens
#pragma unroll
        for (uint32_t c = 0; c < DT / 2; ++c) {
            f16x2 y[8];
            four_values<0>(xv.v[c / 2][2 * (c % 2)], xv.scales, y);
            four_values<1>(xv.v[c / 2][2 * (c % 2) + 1], xv.scales, y);
            Frag16 even, odd;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t lo = __builtin_bit_cast(uint32_t, y[2 * e]), hi = __builtin_bit_cast(uint32_t, y[2 * e + 1]);
                even.w[e] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
                odd.w[e] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
            }
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                acc[i][2 * c] = mfma_fp16(even, p[i], acc[i][2 * c]);
                acc[i][2 * c + 1] = mfma_fp16(odd, p[i], acc[i][2 * c + 1]);
            }
        }
        load_values<D>(xv, at, off);
    }

    if constexpr (TOKEN_WAVES == 1) {
        // register e of a lane: elements (4 g + e) D / 16 .. of row l of each tile
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const uint32_t r = r0 + 16 * i + l;
            if (r >= rows) continue;
            const uint64_t token = sq.first + r / a.group, h = head * a.group + r % a.group;
            if (direct) {
                const float inverse = sum[i] == 0.0f ? 0.0f : 1.0f / sum[i];
                uint16_t *const to = (uint16_t *)a.out + token * a.out_stride + h * D + 4 * g * DT;
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e)
#pragma unroll
                    for (uint32_t d = 0; d < DT; d += 4) {
                        Words2<8> w;
                        w.w[0] = float_elem<T>(acc[i][d][e] * inverse) | float_elem<T>(acc[i][d + 1][e] * inverse) << 16;
                        w.w[1] = float_elem<T>(acc[i][d + 2][e] * inverse) | float_elem<T>(acc[i][d + 3][e] * inverse) << 16;
                        *reinterpret_cast<Words2<8> *>(to + e * DT + d) = w;
                    }
            } else {
                const uint64_t row = ((uint64_t)split * a.c.tokens + token) * a.heads + h;
                const float own = own_factor(m[i], a.c2);
                if (g == 0) a.stat[row] = f32x2{m[i], sum[i] * own};
                float *const to = a.part + row * D + 4 * g * DT;
#pragma unroll
                for (uint32_t e = 0; e < 4; ++e)
#pragma unroll
                    for (uint32_t d = 0; d < DT; d += 4) *reinterpret_cast<f32x4 *>(to + e * DT + d) = f32x4{acc[i][d][e] * own, acc[i][d + 1][e] * own, acc[i][d + 2][e] * own, acc[i][d + 3][e] * own};
            }
        }
    } else {
        // the wavefronts' parts of the same rows meet in LDS, a tile after the other: rows are D + 4 numbers apart
        float own[NR];
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            own[i] = own_factor(m[i], a.c2);
            sum[i] *= own[i];
        }
#pragma unroll
        for (int i = 0; i < NR; ++i)
            if (g == 0) lds_stat[wave * 16 * NR + 16 * i + l] = f32x2{m[i], sum[i]};
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            if (i) __syncthreads();
            float top = LOWEST;
#pragma unroll
            for (uint32_t w = 0; w < TOKEN_WAVES; ++w) top = fmaxf(top, lds_stat[w * 16 * NR + 16 * i + l][0]);
            const float factor = own[i] * __builtin_amdgcn_exp2f((m[i] - top) * a.c2);
            float *const part = lds + (wave * 16 + l) * (D + 4);
#pragma unroll
            for (uint32_t e = 0; e < 4; ++e)
#pragma unroll
                for (uint32_t d = 0; d < DT; d += 4)
                    *reinterpret_cast<f32x4 *>(part + (4 * g + e) * DT + d) = f32x4{acc[i][d][e] * factor, acc[i][d + 1][e] * factor, acc[i][d + 2][e] * factor, acc[i][d + 3][e] * factor};
            __syncthreads();
#pragma unroll
            for (uint32_t x = threadIdx.x; x < 16 * (D / 4); x += 64 * WAVES) {
                const uint32_t in = x / (D / 4), at = 4 * (x % (D / 4)), r = r0 + 16 * i + in;
                if (r >= rows) continue;
                float most = LOWEST, total = 0.0f;
                f32x4 o = {0, 0, 0, 0};
#pragma unroll
                for (uint32_t w = 0; w < TOKEN_WAVES; ++w) most = fmaxf(most, lds_stat[w * 16 * NR + 16 * i + in][0]);
#pragma unroll
                for (uint32_t w = 0; w < TOKEN_WAVES; ++w) {
                    const f32x2 st = lds_stat[w * 16 * NR + 16 * i + in];
                    total += st[1] * __builtin_amdgcn_exp2f((st[0] - most) * a.c2);
                    o += *reinterpret_cast<const f32x4 *>(lds + (w * 16 + in) * (D + 4) + at);
                }
                const uint64_t token = sq.first + r / a.group, h = head * a.group + r % a.group;
                if (direct) {
                    const float inverse = total == 0.0f ? 0.0f : 1.0f / total;
                    Words2<8> w;
                    w.w[0] = float_elem<T>(o[0] * inverse) | float_elem<T>(o[1] * inverse) << 16;
                    w.w[1] = float_elem<T>(o[2] * inverse) | float_elem<T>(o[3] * inverse) << 16;
                    *reinterpret_cast<Words2<8> *>((uint16_t *)a.out + token * a.out_stride + h * D + at) = w;
                } else {
                    const uint64_t row = ((uint64_t)split * a.c.tokens + token) * a.heads + h;
                    if (at == 0) a.stat[row] = f32x2{most, total};
                    *reinterpret_cast<f32x4 *>(a.part + row * D + at) = o;
                }
            }
        }
    }
}

// The parts of a row, joined, where there are several: a wavefront per row, AT_ONCE parts on their way at once.
template <int T, int D, uint32_t AT_ONCE> __global__ void __launch_bounds__(256) attention_join_kernel(const AttentionArgs a, uint32_t block_rows)
{
    constexpr uint32_t PER = D / 64;
    const uint32_t lane = threadIdx.x & 63u;
    const uint32_t r = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);              // row: token, then head
    const Sequence sq = sequence_of(a.c, blockIdx.y);
    const uint32_t n = sq.n < a.max_tokens ? sq.n : a.max_tokens, i = r / a.heads, h = r % a.heads;
    if (i >= n) return;
    const uint32_t in_head = i * a.group + h % a.group;
    const uint32_t parts = granules_of(a, sq, in_head / block_rows * block_rows, block_rows).parts;    // at most 64
    if (parts == 1) return;
    const uint64_t row = (uint64_t)(sq.first + i) * a.heads + h, apart = (uint64_t)a.c.tokens * a.heads;
    const float *const from = a.part + row * D + lane * PER;
    f32x2 st = {LOWEST, 0.0f};
    if (lane < parts) st = a.stat[lane * apart + row];
    float o[PER] = {}, top = LOWEST, factor = 0.0f;
    for (uint32_t z0 = 0; z0 < parts; z0 += AT_ONCE) {
        float x[AT_ONCE][PER];
#pragma unroll
        for (uint32_t z = 0; z < AT_ONCE; ++z) {
            const float *const p = from + (z0 + z < parts ? z0 + z : z0) * apart * D;
#pragma unroll
            for (uint32_t d = 0; d < PER; ++d) x[z][d] = p[d];
        }
        if (z0 == 0) {
            top = st[0];
#pragma unroll
            for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
            factor = __builtin_amdgcn_exp2f((st[0] - top) * a.c2);
        }
#pragma unroll
        for (uint32_t z = 0; z < AT_ONCE; ++z) {
            if (z0 + z >= parts) break;
            const float f = __shfl(factor, (int)(z0 + z));
#pragma unroll
            for (uint32_t d = 0; d < PER; ++d) o[d] += f * x[z][d];
        }
    }
    float total = st[1] * factor;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) total += __shfl_xor(total, d);
    const float inverse = total == 0.0f ? 0.0f : 1.0f / total;
    uint16_t *to = (uint16_t *)a.out + (uint64_t)(sq.first + i) * a.out_stride + (uint64_t)h * D + lane * PER;
    if constexpr (D == 128) *reinterpret_cast<uint32_t *>(to) = float_elem<T>(o[0] * inverse) | float_elem<T>(o[1] * inverse) << 16;
    else *to = (uint16_t)float_elem<T>(o[0] * inverse);
}

// ---- which shape, and how many parts ---------------------------------------------------------
struct Plan { uint32_t nr, row_waves, waves, block_rows, blocks, splits, chunk; bool ordered; };

// Up to 64 rows of a KV head (a token's, a few drafts'): one workgroup has them all, its wavefronts share the tokens.  Eight wavefronts where workgroups are few (one
// sequence, 513 tokens: 6.5 us, 7.5 with four; 131072 tokens: 31 and 33), four else (24 sequences of 35 rows: 21 and 23).  Parts: as many as fill the chip once (eight wavefronts)
// or are resident at once (four; registers leave half as many with two tiles and more of heads of 128), none below four granules a wavefront: 64 sequences of up to 16384 tokens 173 us
// in one part, 147 in two, 152 in eight; one of 131072 47 us in 16 parts, 31 in 32; eight sequences of 64 rows over 8000 41 us in eight parts, 55 in fifteen; 32 of 32 rows over up to
// 4000 35 in two, 40 in four.
//
// More rows: four wavefronts of `nr` tiles each.  The more tiles, the fewer conversions a row costs, but the fewer workgroups there are: the choice goes by the granules that all
// workgroups of three tiles would see, us with one, two and three tiles: 1500 tokens x 32 heads (6000 granules) 43, 48 and 58; 2500 (17000) 89, 80 and 94; 3000 (24000) 115, 106
// and 114; 500 over 8000 (22000) 137, 102 and 110; 4000 (42000) 188, 172 and 157; 8192 (175000) 725, 606 and 540.
// Parts where a row sees much more than comes with the call and workgroups are few: so that they fill the chip once (100 tokens over 8000: 178 us in one part, 42 in nine; 500: 217
// and 103 in four), twice (700 over 8000: 218 in one, 172 in two, 154 in five; 1500 over 12000: 388, 328, and 321 in four) or nearly three times (2048 over 16384: 743 in one, 595 in
// four).  From 450 on the order, longest first, evens them out, and joining the parts costs more than they bring: six chunks of 391 to 1030 tokens over 2159 to
// 6007 323 us in one part, 380 in three; six of 1030 over 6007 644 and 706; 3000 tokens over 9000 399 and 426.
static Plan plan_of(const mmaemu_attention_fp4_args &a)
{
    const uint32_t group = a.heads / a.kv_heads, rows = a.max_tokens * group;
    const uint64_t seen = a.window && (uint64_t)a.window + a.max_tokens < a.max_length ? (uint64_t)a.window + a.max_tokens : a.max_length;
    const uint64_t granules = (seen + 31) / 32, heads = (uint64_t)a.kv_heads * a.sequences;
    Plan p;
    p.ordered = false;
    uint64_t splits, least;
    if (rows <= 64) {
        p.row_waves = 1;
        p.nr = (rows + 15) / 16;
        p.blocks = 1;
        p.waves = heads <= 32 ? 8 : 4;
        splits = heads ? (p.waves == 8 ? 256 : a.dim == 128 && p.nr > 1 ? 512 : 1024) / heads : 1;
        least = 4 * p.waves;
    } else {
        p.row_waves = p.waves = 4;
        const uint64_t triples = heads * ((rows + 191) / 192), all = triples * (seen >= 2ull * a.max_tokens ? granules : (granules + 1) / 2);
        p.nr = all <= 10000 ? 1 : all <= 40000 ? 2 : 3;
        p.blocks = (rows + 64 * p.nr - 1) / (64 * p.nr);
        const uint64_t groups = heads * p.blocks;
        splits = seen < 2ull * a.max_tokens || !groups || groups >= 450 ? 1 : (groups <= 128 ? 512 : groups <= 256 ? 1050 : 1400) / groups;
        least = groups <= 128 ? 4 : groups <= 256 ? 8 : 32;
        p.ordered = a.sequences > 1 && a.sequences <= 64 && seen >= 2ull * a.max_tokens;
    }
    p.block_rows = 16 * p.nr * p.row_waves;
    if (splits > granules / least) splits = granules / least;
    p.splits = splits < 1 ? 1 : splits > 64 ? 64 : (uint32_t)splits;
    p.chunk = (uint32_t)((granules + p.splits - 1) / p.splits);
    if (p.chunk < 1) p.chunk = 1;
    return p;
}

void attention_fp4_name(const mmaemu_attention_fp4_args &a, char *text, size_t size)
{
    if (!a.sequences || !a.tokens || !a.max_tokens) {
        snprintf(text, size, "none");
        return;
    }
    const Plan p = plan_of(a);
    snprintf(text, size, "%s over %u wavefronts, tiles %u, parts %u%s", p.row_waves > 1 ? "rows" : "tokens", p.waves, p.nr, p.splits, p.ordered ? ", longest first" : "");
}

uint64_t attention_fp4_workspace(const mmaemu_attention_fp4_args &a)
{
    if (!a.sequences || !a.tokens || !a.max_tokens) return 0;
    const Plan p = plan_of(a);
    return p.splits > 1 ? (uint64_t)p.splits * a.tokens * a.heads * (a.dim + 2) * 4 : 0;
}

template <int T, int D> static mmaemu_status launch_typed(const AttentionArgs &p, const Plan &plan, hipStream_t s)
{
    const dim3 grid(plan.blocks * p.c.kv_heads, plan.splits, p.c.sequences);
#define MMAEMU_ATTENTION(NR, ROW_WAVES, WAVES) hipLaunchKernelGGL((attention_kernel<T, D, NR, ROW_WAVES, WAVES>), grid, dim3(64 * WAVES), 0, s, p)
#define MMAEMU_ATTENTION_TOKENS(NR)                          \
    do {                                                     \
        if (plan.waves == 8) MMAEMU_ATTENTION(NR, 1, 8);     \
        else MMAEMU_ATTENTION(NR, 1, 4);                     \
    } while (0)
    if (plan.row_waves == 4) {
        if (plan.nr == 1) MMAEMU_ATTENTION(1, 4, 4);
        else if (plan.nr == 2) MMAEMU_ATTENTION(2, 4, 4);
        else MMAEMU_ATTENTION(3, 4, 4);
    } else if (plan.nr == 1) MMAEMU_ATTENTION_TOKENS(1);
    else if (plan.nr == 2) MMAEMU_ATTENTION_TOKENS(2);
    else if (plan.nr == 3) MMAEMU_ATTENTION_TOKENS(3);
    else MMAEMU_ATTENTION_TOKENS(4);
#undef MMAEMU_ATTENTION_TOKENS
#undef MMAEMU_ATTENTION
    MMAEMU_HIP(hipGetLastError());
    if (plan.splits > 1) {
        const uint64_t rows = (uint64_t)p.max_tokens * p.heads;
        const dim3 join((uint32_t)((rows + 3) / 4), p.c.sequences);
        if (plan.splits <= 4) hipLaunchKernelGGL((attention_join_kernel<T, D, 4>), join, dim3(256), 0, s, p, plan.block_rows);
        else if (plan.splits <= 16) hipLaunchKernelGGL((attention_join_kernel<T, D, 16>), join, dim3(256), 0, s, p, plan.block_rows);
        else hipLaunchKernelGGL((attention_join_kernel<T, D, 32>), join, dim3(256), 0, s, p, plan.block_rows);
        MMAEMU_HIP(hipGetLastError());
    }
    return MMAEMU_OK;
}

mmaemu_status launch_attention_fp4(const mmaemu_attention_fp4_args &a, const CacheArgs &c, hipStream_t s)
{
    const Plan plan = plan_of(a);
    AttentionArgs p = {c, a.q, a.out, (float *)a.workspace, nullptr, a.q_stride, a.out_stride, a.heads, a.heads / a.kv_heads, a.max_tokens, a.window, plan.blocks,
                       plan.splits, plan.chunk, (float)(a.scale * 1.4426950408889634)};
    p.ordered = plan.ordered;
    p.stat = (f32x2 *)(p.part + (uint64_t)plan.splits * a.tokens * a.heads * a.dim);
    if (a.type == MMAEMU_BF16) return a.dim == 128 ? launch_typed<MMAEMU_BF16, 128>(p, plan, s) : launch_typed<MMAEMU_BF16, 64>(p, plan, s);
    return a.dim == 128 ? launch_typed<MMAEMU_FP16, 128>(p, plan, s) : launch_typed<MMAEMU_FP16, 64>(p, plan, s);
}

} // namespace mmaemu
