// D = alpha A W^T with W in packed FP4 (E2M1) under group scales: MXFP4 (E8M0 per 32 products) or NVFP4 (UE4M3 per 16), and A in
// BF16 or FP16, or in E4M3 / E5M2 with E8M0 scales per 32.
#include "fp4_operands.hpp"

namespace mmaemu {

constexpr int STREAM_WAVES = 8;

// the activations of one window, and its products
template <int AT, int SF>
__device__ __forceinline__ f32x4 window(const ProductArgs &p, const uint8_t *arow, const uint8_t *sarow, const uint8_t *wrow, const uint8_t *swrow,
                                        uint32_t k0, uint32_t g, f32x4 acc)
{
    const bool in = k0 + 32 * g < p.k;             // k is a multiple of 32: a block is inside as a whole
    u32x4 w = {0, 0, 0, 0};
    if (in) w = *reinterpret_cast<const u32x4 *>(wrow + (k0 + 32 * g) / 2);
    if constexpr (AT == MMAEMU_FP8_E4M3 || AT == MMAEMU_FP8_E5M2) {
        uint32_t sw = 127, sx = 127;
        if (in) {
            sw = swrow[k0 / 32 + g];
            sx = sarow[k0 / 32 + g];
        }
        i32x8 x = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t kx = k0 + 64 * h + 16 * g;
            if (kx < p.k) {
                const u32x4 v = *reinterpret_cast<const u32x4 *>(arow + kx);
#pragma unroll
                for (int q = 0; q < 4; ++q) x[4 * h + q] = (int)v[q];
            }
        }
        return mfma_scaled<AT>(w, sw, x, sx, acc);
    } else {
        Frag16 x[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            x[j].w = u32x4{0, 0, 0, 0};
            if (in) x[j].w = *reinterpret_cast<const u32x4 *>(arow + 2 * (k0 + 32 * g) + 16 * j);
        }
        if constexpr (SF == MMAEMU_SCALE_FORMAT_E8M0) {
            const uint32_t sw = in ? swrow[k0 / 32 + g] : 127u;
            if (AT == MMAEMU_FP16 && __all(fp16_holds(sw))) {
#pragma unroll
                for (int j = 0; j < 4; ++j) acc = mfma_fp16(weights_fp16(w[j], sw), x[j], acc);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (AT == MMAEMU_FP16) {
                        const bool far = sw - 253u < 2u;
                        const Frag16 f = weights_bf16(w[j], far ? sw - 2 : sw);
                        Frag16 hi, lo;
                        split_fp16(x[j], far ? 4.0f : 1.0f, hi, lo);
                        acc = mfma_bf16(f, lo, acc);
                        acc = mfma_bf16(f, hi, acc);
                    } else acc = mfma_bf16(weights_bf16(w[j], sw), x[j], acc);
                }
            }
        } else {
            uint32_t s = 0;
            if (in) s = (swrow[k0 / 16 + 2 * g] & 0x7Fu) | (swrow[k0 / 16 + 2 * g + 1] & 0x7Fu) << 8;
            const f16x2 sh = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(s, 1.0f, 0);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const _Float16 sj = sh[j / 2];
                if (AT == MMAEMU_FP16) acc = mfma_fp16(weights_fp16_by(w[j], f16x2{sj, sj}), x[j], acc);
                else acc = mfma_bf16(weights_bf16_by(w[j], (float)sj), x[j], acc);
            }
        }
        return acc;
    }
}

template <int AT, int SF> __global__ void __launch_bounds__(64 * STREAM_WAVES) stream_kernel(const ProductArgs p)
{
    __shared__ f32x4 part[STREAM_WAVES][64];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, g = lane >> 4;
    const uint32_t n0 = blockIdx.x * 16, m0 = blockIdx.y * 16;
    const uint32_t j = n0 + (lane & 15u) < p.n ? n0 + (lane & 15u) : p.n - 1, i = m0 + (lane & 15u) < p.m ? m0 + (lane & 15u) : p.m - 1;
    const uint8_t *wrow = p.W + (uint64_t)j * (p.k / 2), *swrow = p.SW + (uint64_t)j * (p.k / (SF == MMAEMU_SCALE_FORMAT_E8M0 ? 32 : 16));
    const uint8_t *arow = p.A + (uint64_t)i * p.a_stride, *sarow = p.SA + (uint64_t)i * (p.k / 32);
    f32x4 acc = {0, 0, 0, 0};
    for (uint32_t k0 = 128 * wave; k0 < p.k; k0 += 128 * STREAM_WAVES) acc = window<AT, SF>(p, arow, sarow, wrow, swrow, k0, g, acc);
    part[wave][lane] = acc;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 1; w < STREAM_WAVES; ++w) acc += part[w][lane];
    with_output_type(p.d_type, [&](auto dt) { store_outputs<dt.value>(p, m0 + (lane & 15u), n0 + 4 * g, acc); });
}

template <int AT, int SF> static mmaemu_status launch_product(const ProductArgs &p, hipStream_t s)
{
    hipLaunchKernelGGL((stream_kernel<AT, SF>), dim3((p.n + 15) / 16, (p.m + 15) / 16), dim3(64 * STREAM_WAVES), 0, s, p);
    MMAEMU_HIP(hipGetLastError());
    return MMAEMU_OK;
}

mmaemu_status launch_matmul_fp4(const void *A, const void *SA, const void *W, const void *SW, void *D, uint32_t m, uint32_t n, uint32_t k,
                                uint64_t a_stride, uint64_t d_stride, uint32_t a_type, uint32_t d_type, uint32_t scale_format, float alpha, hipStream_t s)
{
    const bool bytes = a_type == MMAEMU_FP8_E4M3 || a_type == MMAEMU_FP8_E5M2;
    const ProductArgs p = {(const uint8_t *)A, (const uint8_t *)SA, (const uint8_t *)W, (const uint8_t *)SW, D, a_stride * (bytes ? 1 : 2), d_stride, m, n, k,
                           d_type, alpha};
    if (m >= 256) return launch_tiled(p, a_type, scale_format, s);
    if (a_type == MMAEMU_FP8_E4M3) return launch_product<MMAEMU_FP8_E4M3, MMAEMU_SCALE_FORMAT_E8M0>(p, s);
    if (a_type == MMAEMU_FP8_E5M2) return launch_product<MMAEMU_FP8_E5M2, MMAEMU_SCALE_FORMAT_E8M0>(p, s);
    if (scale_format == MMAEMU_SCALE_FORMAT_E8M0)
        return a_type == MMAEMU_BF16 ? launch_product<MMAEMU_BF16, MMAEMU_SCALE_FORMAT_E8M0>(p, s) : launch_product<MMAEMU_FP16, MMAEMU_SCALE_FORMAT_E8M0>(p, s);
    return a_type == MMAEMU_BF16 ? launch_product<MMAEMU_BF16, MMAEMU_SCALE_FORMAT_UE4M3>(p, s) : launch_product<MMAEMU_FP16, MMAEMU_SCALE_FORMAT_UE4M3>(p, s);
}

} // namespace mmaemu
