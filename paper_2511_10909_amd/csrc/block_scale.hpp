// Device helpers of the block-scaled operators: elements of 16 and 32 bits in vectors of eight, the scale of a block and its
// codes.  The conversions to and from E4M3, E5M2 and E2M1 are gfx950's own instructions (round to nearest even, subnormal
// codes included); what they leave undefined for a format without infinities (values above the largest) is cut off before them.
#pragma once
#include "common.hpp"

namespace mmaemu {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// Words at any address that its elements' alignment allows: the memory system takes unaligned vector accesses whole.
template <int ALIGN> struct __attribute__((packed, aligned(ALIGN))) Words4 { uint32_t w[4]; };
template <int ALIGN> struct __attribute__((packed, aligned(ALIGN))) Words2 { uint32_t w[2]; };

__device__ __forceinline__ float word_float(uint32_t b) { return __uint_as_float(b); }

template <int T> __device__ __forceinline__ float elem_float(uint32_t bits)      // one 16-bit element
{
    if (T == MMAEMU_BF16) return __uint_as_float(bits << 16);
    const uint16_t h = (uint16_t)bits;
    return (float)__builtin_bit_cast(_Float16, h);
}
template <int T> __device__ __forceinline__ uint32_t float_elem(float x)          // rounded to nearest even
{
    if (T == MMAEMU_BF16) return __builtin_bit_cast(uint16_t, (__bf16)x);
    if (T == MMAEMU_FP16) return __builtin_bit_cast(uint16_t, (_Float16)x);
    return __float_as_uint(x);
}
constexpr int elem_bytes(int t) { return t == MMAEMU_FP32 ? 4 : 2; }

// Eight consecutive elements as they lie in memory (one or two 16-byte accesses).
template <int T> struct Raw8 { uint32_t w[T == MMAEMU_FP32 ? 8 : 4]; };

template <int T> __device__ __forceinline__ Raw8<T> load8(const void *base, uint64_t at)
{
    Raw8<T> r;
    typedef Words4<elem_bytes(T)> W;
    const W *p = reinterpret_cast<const W *>((const char *)base + at * elem_bytes(T));
#pragma unroll
    for (int h = 0; h < (T == MMAEMU_FP32 ? 2 : 1); ++h) {
        const W v = p[h];
#pragma unroll
        for (int q = 0; q < 4; ++q) r.w[4 * h + q] = v.w[q];
    }
    return r;
}
// the first `count` (0 .. 8) of them, the rest zero
template <int T> __device__ __forceinline__ Raw8<T> load_some(const void *base, uint64_t at, int count)
{
    Raw8<T> r;
#pragma unroll
    for (int q = 0; q < (T == MMAEMU_FP32 ? 8 : 4); ++q) r.w[q] = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < count) {
            if (T == MMAEMU_FP32) r.w[i] = ((const uint32_t *)base)[at + i];
            else r.w[i / 2] |= (uint32_t)((const uint16_t *)base)[at + i] << (16 * (i % 2));
        }
    return r;
}
template <int T> __device__ __forceinline__ void store8(void *base, uint64_t at, const Raw8<T> &r)
{
    typedef Words4<elem_bytes(T)> W;
    W *p = reinterpret_cast<W *>((char *)base + at * elem_bytes(T));
#pragma unroll
    for (int h = 0; h < (T == MMAEMU_FP32 ? 2 : 1); ++h) {
        W v;
#pragma unroll
        for (int q = 0; q < 4; ++q) v.w[q] = r.w[4 * h + q];
        p[h] = v;
    }
}
template <int T> __device__ __forceinline__ void store_some(void *base, uint64_t at, const Raw8<T> &r, int count)
{
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < count) {
            if (T == MMAEMU_FP32) ((uint32_t *)base)[at + i] = r.w[i];
            else ((uint16_t *)base)[at + i] = (uint16_t)(r.w[i / 2] >> (16 * (i % 2)));
        }
}
template <int T> __device__ __forceinline__ float get8(const Raw8<T> &r, int i)
{
    if (T == MMAEMU_FP32) return __uint_as_float(r.w[i]);
    if (T == MMAEMU_BF16) return __uint_as_float(i % 2 ? r.w[i / 2] & 0xFFFF0000u : r.w[i / 2] << 16);
    return elem_float<T>((r.w[i / 2] >> (16 * (i % 2))) & 0xFFFFu);
}
template <int T> __device__ __forceinline__ Raw8<T> round8(const float (&v)[8])
{
    Raw8<T> r;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        if (T == MMAEMU_FP32) {
            r.w[i] = __float_as_uint(v[i]);
            r.w[i + 1] = __float_as_uint(v[i + 1]);
        } else r.w[i / 2] = float_elem<T>(v[i]) | float_elem<T>(v[i + 1]) << 16;
    }
    return r;
}

// Binary64 to binary32 such that a later rounding to a few bits comes out as if taken from the binary64 value: cut toward
// zero, the last bit set where anything was lost.  Values that are subnormal in binary32 are rounded there: zeros to E2M1, E4M3 and
// FP16, but not to BF16, which reaches as far down.
__device__ __forceinline__ float to_float_odd(double x)
{
    uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t low = (uint32_t)b & 0x1FFFFFFFu;
    b = (b & ~0x1FFFFFFFull) | (low ? 0x20000000ull : 0ull);
    return (float)__builtin_bit_cast(double, b);
}

// The same for all magnitudes: below binary32's least normal number its pattern counts units of 2^-149.
__device__ __forceinline__ float to_float_odd_subnormal(double x)
{
    const double a = __builtin_fabs(x);
    if (a >= 0x1p-126) return to_float_odd(x);
    const double units = a * 0x1p149;              // exact, below 2^23
    const uint32_t whole = (uint32_t)units;
    return __builtin_copysignf(__uint_as_float(whole | ((double)whole != units ? 1u : 0u)), (float)x);
}

// ---- a block's E8M0 scale ---------------------------------------------------------------
// Largest magnitude amax (binary32 pattern, sign cleared): floor rule, the exponent at which amax and the element type's
// largest power of two (2^EMAX) meet; fit rule, one more where amax exceeds the type's largest number, whose mantissa
// field is TOPMAN.  Blocks of zeros and of numbers too small for the scale take code 0; a block with an infinity or a
// NaN code 0xFF.
template <int EMAX, uint32_t TOPMAN> __device__ __forceinline__ uint32_t e8m0_code(uint32_t amax, bool fit)
{
    if (amax >= 0x7F800000u) return 0xFFu;
    const int e = (int)(amax >> 23) - EMAX + (fit && (amax & 0x7FFFFFu) > TOPMAN ? 1 : 0);
    return e < 0 ? 0u : (uint32_t)e;
}
// 2^(127 - code), which takes a block to its elements' range (code at most 253); 0 for the NaN code: no element is read then
__device__ __forceinline__ float e8m0_inverse(uint32_t code) { return code == 0xFFu ? 0.0f : __uint_as_float((254u - code) << 23); }

// ---- reductions over lanes by DPP ---------------------------------------------------------
template <int CTRL> __device__ __forceinline__ uint32_t dpp_max(uint32_t x)
{
    const uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, CTRL, 0xF, 0xF, false);
    return o > x ? o : x;
}
__device__ __forceinline__ uint32_t max_of_pair(uint32_t x) { return dpp_max<0xB1>(x); }                    // lanes 2i, 2i + 1
__device__ __forceinline__ uint32_t max_of_quad(uint32_t x) { return dpp_max<0x4E>(dpp_max<0xB1>(x)); }     // lanes 4i .. 4i + 3

template <int CTRL, int ROWS> __device__ __forceinline__ double dpp_add(double x)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROWS, 0xF, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, ROWS, 0xF, false);
    return x + __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
// sum over the wavefront, in every lane
__device__ __forceinline__ double wave_sum(double x)
{
    x = dpp_add<0x111, 0xF>(x);                    // row_shr 1, 2, 4, 8: lane 15 of each row of 16 holds the row's sum
    x = dpp_add<0x112, 0xF>(x);
    x = dpp_add<0x114, 0xF>(x);
    x = dpp_add<0x118, 0xF>(x);
    x = dpp_add<0x142, 0xA>(x);                    // row_bcast15 into rows 1 and 3
    x = dpp_add<0x143, 0xC>(x);                    // row_bcast31 into rows 2 and 3: lane 63 holds the sum
    const uint64_t b = __builtin_bit_cast(uint64_t, x);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, 63), hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), 63);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

} // namespace mmaemu
