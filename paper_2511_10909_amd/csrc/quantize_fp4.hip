// Weights to FP4 (E2M1) with group scales: MXFP4 (E8M0 per 32 elements) or NVFP4 (UE4M3 per 16, and one binary32 scale for
// the tensor), packed two to a byte, with the values that codes and scales stand for on request.
//
//   E8M0:  code by the scale rule from the group's largest magnitude; elements RNE_E2M1(x 2^(127 - code)), saturated
//   UE4M3: scale s = RNE_E4M3(min(448, amax / (6 t))), t the tensor's scale; elements RNE_E2M1(x / (s t)), saturated
//          (s = 0: zeros); codes are those of the exact quotients
//
// Bound by memory: 2 bytes read and 0.53 (values: 2.53) written per 16-bit element.  A thread holds eight consecutive
// elements: 16 bytes in, 4 of codes out, a group's maximum over two or four lanes.  4096 x 4096 BF16 to MXFP4 with values: 13.3 us, 5.7 TB/s;
// 11003 x 5000 binary32 to NVFP4 with values: 98 us, 4.8 TB/s (100.5 with every quotient in binary64).  Codes and scales alone: 8192 x 28672
// BF16 to MXFP4 110 us, 5.4 TB/s, to NVFP4 162, 3.7 (with values 187 and 241); 11003 x 5000 binary32 to NVFP4 54 us, 4.7 TB/s.
#include "block_scale.hpp"

namespace mmaemu {

struct QuantArgs {
    const void *x;
    uint8_t *codes, *scales;
    void *values;
    uint64_t rows, x_stride;
    uint32_t cols, vectors;                        // vectors: of eight elements, of a row padded to whole blocks of 32
    uint32_t fit;
    float tensor_scale;
    double inverse_6t;                             // 1 / (6 tensor_scale), rounded
};

constexpr int QUANT_UNROLL = 4;

__device__ __forceinline__ uint32_t pack_fp4(const float (&f)[8])
{
    uint32_t q = 0;
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[0], f[1], 1.0f, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[2], f[3], 1.0f, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[4], f[5], 1.0f, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, f[6], f[7], 1.0f, 3);
}

// x / d, correctly rounded: the product with the rounded inverse, corrected by its exact remainder
__device__ __forceinline__ double quotient(double x, double d, double inverse)
{
    const double p = x * inverse;
    return __builtin_fma(__builtin_fma(-p, d, x), inverse, p);
}

template <int T, bool UE4M3>
__device__ __forceinline__ void quantize_vector(const QuantArgs &a, uint64_t row, uint32_t v, const Raw8<T> &x)
{
    const int left = (int)a.cols - (int)(8 * v);
    float f[8];
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        f[i] = get8<T>(x, i);
        const uint32_t b = magnitude(f[i]);
        amax = b > amax ? b : amax;
    }
    const uint64_t at = row * a.vectors + v;
    uint32_t q = 0;
    bool nan;
    float out[8], scale = 0.0f;
    if constexpr (!UE4M3) {
        const uint32_t code = e8m0_code<2, 0x400000u>(max_of_quad(amax), a.fit);
        nan = code == 0xFFu;
        const float inv = e8m0_inverse(code);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] *= inv;
        if ((v & 3u) == 0) a.scales[at / 4] = (uint8_t)code;
        if (!nan) q = pack_fp4(f);
        if (a.values) {
            const float unit = __uint_as_float(code << 23);            // (the conversion reads exponent field 0 as 2^-127)
            const f32x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, unit, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, unit, 1),
                        p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, unit, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, unit, 3);
            out[0] = p0[0]; out[1] = p0[1]; out[2] = p1[0]; out[3] = p1[1]; out[4] = p2[0]; out[5] = p2[1]; out[6] = p3[0]; out[7] = p3[1];
        }
    } else {
        amax = max_of_pair(amax);
        nan = amax >= 0x7F800000u;
        const double t = (double)a.tensor_scale;
        float s = to_float_odd(quotient((double)__uint_as_float(amax), 6.0 * t, a.inverse_6t));
        s = s < 448.0f ? s : 448.0f;
        const uint32_t code = nan ? 0x7Fu : (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(s, 0.0f, 0, false) & 0xFFu;
        scale = __builtin_amdgcn_cvt_f32_fp8((int)code, 0);
        const double unit = (double)scale * t;                         // exact: 4 + 24 bits
        if ((v & 1u) == 0) a.scales[at / 2] = (uint8_t)code;
        if (!nan) {
            // Binary32 quotients are within 2^-22: where 2^-20 on either side gives the same codes, those are the quotients' own.  Where
            // it does not (next to a border between two codes: one vector in 10^5), and for units that binary32's inverse does not hold, binary64.
            const float u = (float)unit;
            const float inv = code == 0 ? 0.0f : __builtin_amdgcn_rcpf(u);
            float lo[8], hi[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float c = f[i] * inv;
                lo[i] = __builtin_amdgcn_fmed3f(c * (1.0f - 0x1p-20f), -6.0f, 6.0f);
                hi[i] = __builtin_amdgcn_fmed3f(c * (1.0f + 0x1p-20f), -6.0f, 6.0f);
            }
            q = pack_fp4(lo);
            const bool held = code == 0 || (u >= 0x1p-126f && u <= 0x1p125f);
            if (!held || q != pack_fp4(hi)) {
                const double inverse = 1.0 / unit;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float c = __builtin_amdgcn_fmed3f(to_float_odd(quotient((double)f[i], unit, inverse)), -6.0f, 6.0f);
                    lo[i] = __builtin_copysignf(c, f[i]);              // (the remainder's sum turns -0 into +0)
                }
                q = pack_fp4(lo);
            }
        }
        if (a.values) {
            const f32x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 1),
                        p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 3);
            const float e[8] = {p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
            const bool low = T == MMAEMU_BF16 && a.tensor_scale < 0x1p-116f;           // (the least element and scale make 2^-10)
            if (__builtin_expect(low, 0)) {
#pragma unroll
                for (int i = 0; i < 8; ++i) out[i] = to_float_odd_subnormal((double)(e[i] * scale) * (double)a.tensor_scale);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float es = e[i] * scale;                     // exact: 2 + 4 bits, and 24 more with the tensor's scale
                    out[i] = T == MMAEMU_FP32 ? es * a.tensor_scale : to_float_odd((double)es * (double)a.tensor_scale);
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (nan) out[i] = __uint_as_float(0x7FC00000u);
        }
    }
    struct __attribute__((packed, aligned(1))) Word { uint32_t w; } word = {q};
    *reinterpret_cast<Word *>(a.codes + 4 * at) = word;
    if (a.values && left > 0) {
        const Raw8<T> r = round8<T>(out);
        if (left >= 8) store8<T>(a.values, row * a.cols + 8ull * v, r);
        else store_some<T>(a.values, row * a.cols + 8ull * v, r, left);
    }
}

template <int T, bool UE4M3> __global__ void __launch_bounds__(256) quantize_fp4_kernel(const QuantArgs a)
{
    // the workgroup's first vector as row and column, by one division of uniform numbers; the threads' by 32-bit ones
    const uint64_t first = (uint64_t)blockIdx.x * (256 * QUANT_UNROLL);
    const uint64_t row0 = first / a.vectors;
    const uint32_t col0 = (uint32_t)(first - row0 * a.vectors);
    uint64_t row[QUANT_UNROLL];
    uint32_t v[QUANT_UNROLL];
    Raw8<T> x[QUANT_UNROLL];
#pragma unroll
    for (int u = 0; u < QUANT_UNROLL; ++u) {
        const uint32_t p = col0 + u * 256 + threadIdx.x, q = p / a.vectors;
        row[u] = row0 + q;
        v[u] = p - q * a.vectors;
        const int left = (int)a.cols - (int)(8 * v[u]);
        if (row[u] < a.rows) x[u] = left >= 8 ? load8<T>(a.x, row[u] * a.x_stride + 8ull * v[u]) : load_some<T>(a.x, row[u] * a.x_stride + 8ull * v[u], left);
    }
#pragma unroll
    for (int u = 0; u < QUANT_UNROLL; ++u)
        if (row[u] < a.rows) quantize_vector<T, UE4M3>(a, row[u], v[u], x[u]);
}

template <int T> static void launch_quant(const QuantArgs &a, bool ue4m3, hipStream_t s)
{
    const dim3 grid((uint32_t)((a.rows * a.vectors + 256 * QUANT_UNROLL - 1) / (256 * QUANT_UNROLL)));
    if (ue4m3) hipLaunchKernelGGL((quantize_fp4_kernel<T, true>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((quantize_fp4_kernel<T, false>), grid, dim3(256), 0, s, a);
}

mmaemu_status launch_quantize_fp4(const void *x, void *codes, void *scales, void *values, uint64_t rows, uint32_t cols, uint64_t x_stride,
                                  uint32_t type, uint32_t scale_format, uint32_t scale_rule, float tensor_scale, hipStream_t s)
{
    const bool ue4m3 = scale_format == MMAEMU_SCALE_FORMAT_UE4M3;
    const uint32_t vectors = (cols + 31) / 32 * 4, eb = type == MMAEMU_FP32 ? 4 : 2;
    const uint64_t most = (1ull << 33) / vectors;                      // rows of one launch: its threads count in 32 bits
    for (uint64_t r0 = 0; r0 < rows; r0 += most) {
        const QuantArgs a = {(const char *)x + r0 * x_stride * eb, (uint8_t *)codes + r0 * vectors * 4, (uint8_t *)scales + r0 * (vectors / (ue4m3 ? 2 : 4)),
                             values ? (char *)values + r0 * cols * eb : nullptr, rows - r0 < most ? rows - r0 : most, x_stride, cols, vectors,
                             scale_rule == MMAEMU_SCALE_RULE_FIT, tensor_scale, 1.0 / (6.0 * (double)tensor_scale)};
        switch (type) {
        case MMAEMU_BF16: launch_quant<MMAEMU_BF16>(a, ue4m3, s); break;
        case MMAEMU_FP16: launch_quant<MMAEMU_FP16>(a, ue4m3, s); break;
        default: launch_quant<MMAEMU_FP32>(a, ue4m3, s); break;
        }
        MMAEMU_HIP(hipGetLastError());
    }
    return MMAEMU_OK;
}

} // namespace mmaemu
