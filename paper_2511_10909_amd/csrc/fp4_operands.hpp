// Operands of the products with packed FP4 weights: what a lane of the 16 x 16 matrix instructions holds, from memory as it
// lies.  The weights are the first operand and the activations the second, so that a lane ends with four consecutive
// outputs of one token.
//
// A window is 128 products of a row.  Lane l holds weight row l % 16, codes 32 g .. 32 g + 31 of the window with g = l / 16:
// sixteen bytes, all under one E8M0 scale or two UE4M3 scales.
//   8-bit activations, v_mfma_scale_f32_16x16x128_f8f6f4: token l % 16, k = 16 g .. + 15 and 64 + 16 g .. + 15; the scale
//     operand carries the code of block g in its low byte.
//   16-bit activations, four v_mfma_f32_16x16x32: the sum does not mind which k an instruction takes, so instruction j takes
//     k = 32 g + 8 j + i from lane l (i = 0 .. 7): both operands are then contiguous in memory and every lane stays in one block.
#pragma once
#include "block_scale.hpp"
#include <type_traits>

// for lambdas of the kernels: one that is not inlined holds all that it names in scratch memory
#define MMAEMU_INLINE __attribute__((always_inline))

namespace mmaemu {

// Weights of 16-bit activations are brought to the activations' type, scale included.  That is exact: E2M1 2^(code - 127) is
// a BF16 number (from magnitude 2^128 on an infinity, as in binary32), E2M1 UE4M3 has six significant bits and lies in
// 2^-10 .. 2688, within FP16.  FP16 weights under E8M0 scales are exact for codes 104 .. 140 (2^-23 .. 2^13); other codes
// take the BF16 way, with the activations split into two BF16 numbers (their eleven bits fit two times eight).
__device__ __forceinline__ bool fp16_holds(uint32_t code) { return code - 104u <= 36u; }

struct Frag16 { u32x4 w; };                        // eight 16-bit elements

__device__ __forceinline__ Frag16 weights_bf16(uint32_t codes, uint32_t e8m0)
{
    const float s = __uint_as_float(e8m0 << 23);   // (field 0 is read as 2^-127, field 255 as NaN)
    Frag16 f;
    f.w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0));
    f.w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1));
    f.w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2));
    f.w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3));
    return f;
}
__device__ __forceinline__ Frag16 weights_fp16(uint32_t codes, uint32_t e8m0)
{
    const float s = __uint_as_float(e8m0 << 23);
    Frag16 f;
    f.w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, 0));
    f.w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, 1));
    f.w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, 2));
    f.w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, s, 3));
    return f;
}
// under a UE4M3 scale, given in binary32 (BF16) or twice in FP16
__device__ __forceinline__ Frag16 weights_bf16_by(uint32_t codes, float s)
{
    Frag16 f;
    const f32x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 1),
                p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, 1.0f, 3);
    f.w[0] = float_elem<MMAEMU_BF16>(p0[0] * s) | float_elem<MMAEMU_BF16>(p0[1] * s) << 16;
    f.w[1] = float_elem<MMAEMU_BF16>(p1[0] * s) | float_elem<MMAEMU_BF16>(p1[1] * s) << 16;
    f.w[2] = float_elem<MMAEMU_BF16>(p2[0] * s) | float_elem<MMAEMU_BF16>(p2[1] * s) << 16;
    f.w[3] = float_elem<MMAEMU_BF16>(p3[0] * s) | float_elem<MMAEMU_BF16>(p3[1] * s) << 16;
    return f;
}
__device__ __forceinline__ Frag16 weights_fp16_by(uint32_t codes, f16x2 s)
{
    Frag16 f;
    f.w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 1.0f, 0) * s);
    f.w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 1.0f, 1) * s);
    f.w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 1.0f, 2) * s);
    f.w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, 1.0f, 3) * s);
    return f;
}

// A quarter of the scale that an E8M0 code stands for (255: NaN).
__device__ __forceinline__ float quarter_scale(uint32_t e8m0)
{
    return __uint_as_float(e8m0 == 255u ? 0x7FC00000u : e8m0 > 2u ? (e8m0 - 2u) << 23 : 0x00100000u << e8m0);
}
// FP16's second way: weights in BF16.  Those of codes 253 and 254 reach 2^128, and an infinity must not meet the zeros among the activations'
// smaller parts.  Where a lane of the wavefront holds such a code (`far`, the same in all lanes: lane r holds weight row r and token r, and
// an instruction multiplies each with all of the other), every lane takes its weights at a quarter, which is exact down to code 0, and its
// activations four times.
__device__ __forceinline__ bool any_far(uint32_t code) { return __any(code - 253u < 2u); }
__device__ __forceinline__ Frag16 weights_second_way(uint32_t codes, uint32_t e8m0, bool far)
{
    return far ? weights_bf16_by(codes, quarter_scale(e8m0)) : weights_bf16(codes, e8m0);
}
// eight FP16 activations, times 1 or 4, as sums of two BF16 numbers each
__device__ __forceinline__ void split_fp16(const Frag16 &x, float factor, Frag16 &hi, Frag16 &lo)
{
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float a = elem_float<MMAEMU_FP16>(x.w[q] & 0xFFFFu) * factor, b = elem_float<MMAEMU_FP16>(x.w[q] >> 16) * factor;
        const uint32_t ha = float_elem<MMAEMU_BF16>(a), hb = float_elem<MMAEMU_BF16>(b);
        const float ra = a - __uint_as_float(ha << 16), rb = b - __uint_as_float(hb << 16);
        hi.w[q] = ha | hb << 16;
        // (an infinity leaves no remainder: infinity minus itself is NaN)
        lo.w[q] = (magnitude(a) >= 0x7F800000u ? 0u : float_elem<MMAEMU_BF16>(ra)) | (magnitude(b) >= 0x7F800000u ? 0u : float_elem<MMAEMU_BF16>(rb)) << 16;
    }
}

__device__ __forceinline__ f32x4 mfma_bf16(const Frag16 &a, const Frag16 &b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.w), __builtin_bit_cast(bf16x8, b.w), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_fp16(const Frag16 &a, const Frag16 &b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a.w), __builtin_bit_cast(f16x8, b.w), c, 0, 0, 0);
}
// AT: MMAEMU_FP8_E4M3 or MMAEMU_FP8_E5M2 (formats 0 and 1 of the instruction; 4 is E2M1).
// Of eight consecutive products the instruction keeps 13 bits below the largest, then adds in 24.  That is fewer than binary32's, and taken
// for its rate: 8192^3 E4M3 389 us; the same operands brought to BF16, which would keep 24 throughout, are the BF16 kernel's 789.  Binary32
// outputs of 256 to 8192 products are 5e-6 to 9e-6 (relative, in the mean square) from the exact ones, where sums in binary32 are 4e-8;
// BF16 and FP16 outputs are as near as those, 1.7e-3 and 2.1e-4, and one in some hundred falls on the other side of its own rounding.
template <int AT> __device__ __forceinline__ f32x4 mfma_scaled(u32x4 w, uint32_t sw, const i32x8 &x, uint32_t sx, f32x4 c)
{
    const i32x8 a = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, x, c, 4, AT == MMAEMU_FP8_E5M2 ? 1 : 0, 0, (int)sw, 0, (int)sx);
}

__device__ __forceinline__ uint32_t lds_address(const uint8_t *p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t *)p; }

// Sixteen bytes per lane from memory to LDS, to + 16 lane.  By hand: before a read the compiler waits for every copy that it
// knows of, as it cannot tell the buffers apart.  No register is written, and the address is read as the copy is issued.
__device__ __forceinline__ void copy_to_lds(const uint8_t *from, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(to) : "memory");
}

// the same from a uniform base
__device__ __forceinline__ void copy_to_lds(const uint8_t *base, uint32_t from, uint32_t to)
{
    // (uniform in any case: the compiler may hold them in vector registers)
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)base), hi = __builtin_amdgcn_readfirstlane((uint32_t)((uintptr_t)base >> 32));
    base = (const uint8_t *)((uintptr_t)hi << 32 | lo);
    to = __builtin_amdgcn_readfirstlane(to);
    // (five wait states between a vector instruction that may have written the base and its use)
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(from), "s"(base), "s"(to) : "memory");
}
// one aligned word per lane, to + 4 lane
__device__ __forceinline__ void copy_word_to_lds(const uint8_t *from, uint32_t to)
{
    to = __builtin_amdgcn_readfirstlane(to);
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(from), "s"(to) : "memory");
}

// Reads of sixteen bytes per lane serve the lanes 0 - 3, 12 - 15, 20 - 27 together, then 4 - 11, 16 - 19, 28 - 31, and so the upper 32; the
// sixteen have to differ in their place within 256 bytes (found with the conflict counter).  Lane l reads row l % 16, and its group of
// lanes l / 16 picks the 16-byte chunk: chunk c of row r is stored at c ^ lds_rotation<chunks of a row>(r).
template <int CHUNKS> __device__ __forceinline__ constexpr uint32_t lds_rotation(uint32_t r)
{
    const uint32_t r1 = (r >> 1) & 1, r2 = (r >> 2) & 1, r3 = (r >> 3) & 1;
    if (CHUNKS == 16) return (r2 ^ r3) << 3 | r3 << 2 | (r & 3);
    if (CHUNKS == 8) return (r2 ^ r3) << 2 | r3 << 1 | r1;
    if (CHUNKS == 4) return (r >> 1) & 3;
    return r3;                                     // two: 32 bytes, read by eights
}

struct ProductArgs {
    const uint8_t *A, *SA, *W, *SW;
    void *D;
    uint64_t a_stride, d_stride;                   // of A in bytes, of D in elements
    uint32_t m, n, k;
    uint32_t d_type;
    float alpha;
};

// the kernel for many rows of A (matmul_fp4_tiled.hip)
mmaemu_status launch_tiled(const ProductArgs &p, uint32_t a_type, uint32_t scale_format, hipStream_t s);
const char *tiled_name(uint32_t m, uint32_t n, uint32_t k, uint32_t a_type, uint32_t scale_format);

// four consecutive outputs of one token, columns j .. j + 3, in type DT
template <int DT> __device__ __forceinline__ void store_outputs(const ProductArgs &p, uint32_t i, uint32_t j, f32x4 v)
{
    if (i >= p.m || j >= p.n) return;
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] *= p.alpha;
    const uint64_t at = (uint64_t)i * p.d_stride + j;
    const uint32_t left = p.n - j;
    if constexpr (DT == MMAEMU_FP32) {
        float *d = (float *)p.D + at;
        if (left >= 4) {
            Words4<4> o;
#pragma unroll
            for (int q = 0; q < 4; ++q) o.w[q] = __float_as_uint(v[q]);
            *reinterpret_cast<Words4<4> *>(d) = o;
        } else {
            d[0] = v[0];
            if (left > 1) d[1] = v[1];
            if (left > 2) d[2] = v[2];
        }
    } else {
        uint16_t *d = (uint16_t *)p.D + at;
        if (left >= 4) {
            Words2<2> o;
            o.w[0] = float_elem<DT>(v[0]) | float_elem<DT>(v[1]) << 16;
            o.w[1] = float_elem<DT>(v[2]) | float_elem<DT>(v[3]) << 16;
            *reinterpret_cast<Words2<2> *>(d) = o;
        } else {
            d[0] = (uint16_t)float_elem<DT>(v[0]);
            if (left > 1) d[1] = (uint16_t)float_elem<DT>(v[1]);
            if (left > 2) d[2] = (uint16_t)float_elem<DT>(v[2]);
        }
    }
}
// f<DT>() for the output type of a launch
template <class F> __device__ __forceinline__ void with_output_type(uint32_t d_type, F f)
{
    if (d_type == MMAEMU_BF16) f(std::integral_constant<int, MMAEMU_BF16>());
    else if (d_type == MMAEMU_FP16) f(std::integral_constant<int, MMAEMU_FP16>());
    else f(std::integral_constant<int, MMAEMU_FP32>());
}

} // namespace mmaemu
