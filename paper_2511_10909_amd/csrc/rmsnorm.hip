// Root-mean-square norm with the residual's addition and an output in 8 bits with a power-of-two scale per 32 elements.
//
//   h = RN_type(x + residual)                                  (the residual stream, held in its type)
//   y = RN_fp32(h / sqrt(mean(h^2) + eps) * weight)
//   per 32 elements of y: code E8M0 by the scale rule (block_scale.hpp), elements RNE(y 2^(127 - code)), saturated
//
// Bound by memory: per 16-bit element 2 + 2 bytes read, 2 + 1 written.  The sum of squares, the root and the product are
// binary64: its vector rate is that of binary32 on this chip, so it costs nothing beside the traffic, no row of binary32
// numbers overflows or vanishes in its squares, and the result does not depend on the order of the sum but for one in
// 2^28 elements or so (the one rounding to binary32 that could fall either way).
//
// A thread holds vectors of eight consecutive elements of a row, vector t + i TPR for i < NV (TPR threads per row), so
// that every access is 16 bytes (8 of codes) and four lanes hold one block; nothing is read twice.
#include "block_scale.hpp"

namespace mmaemu {

struct NormArgs {
    const void *x, *residual, *weight;
    void *residual_out;
    uint8_t *codes, *scales;
    uint64_t rows, x_stride, residual_stride;
    uint32_t cols, vectors;                        // vectors: of eight elements, of a row padded to whole blocks
    uint32_t e5m2, fit;
    double eps;
};

// h of one vector, and its store
template <int T> __device__ __forceinline__ Raw8<T> norm_input(const NormArgs &a, uint64_t row, uint32_t v)
{
    const int left = (int)a.cols - (int)(8 * v);
    const uint64_t at = row * a.x_stride + 8ull * v, ar = row * a.residual_stride + 8ull * v;
    Raw8<T> x = left >= 8 ? load8<T>(a.x, at) : load_some<T>(a.x, at, left);
    if (a.residual) {
        const Raw8<T> r = left >= 8 ? load8<T>(a.residual, ar) : load_some<T>(a.residual, ar, left);
        float s[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] = get8<T>(x, i) + get8<T>(r, i);
        x = round8<T>(s);
        if (a.residual_out) {
            if (left >= 8) store8<T>(a.residual_out, ar, x);
            else store_some<T>(a.residual_out, ar, x, left);
        }
    }
    return x;
}

template <int T> __device__ __forceinline__ double squares(const Raw8<T> &h, double s)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double d = (double)get8<T>(h, i);
        s = __builtin_fma(d, d, s);
    }
    return s;
}

// codes and scale of one vector; the four lanes of a block are all here
template <int T, int TW>
__device__ __forceinline__ void norm_output(const NormArgs &a, uint64_t row, uint32_t v, const Raw8<T> &h, double r)
{
    const int left = (int)a.cols - (int)(8 * v);
    Raw8<TW> w;
    if (a.weight) w = left >= 8 ? load8<TW>(a.weight, 8ull * v) : load_some<TW>(a.weight, 8ull * v, left);
    float y[8];
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        double d = (double)get8<T>(h, i) * r;
        if (a.weight) d *= (double)get8<TW>(w, i);
        y[i] = i < left ? (float)d : 0.0f;         // (beyond the row h is zero, but r may be infinite)
        const uint32_t b = magnitude(y[i]);
        amax = b > amax ? b : amax;
    }
    amax = max_of_quad(amax);
    const uint32_t code = a.e5m2 ? e8m0_code<15, 0x600000u>(amax, a.fit) : e8m0_code<8, 0x600000u>(amax, a.fit);
    const float inv = e8m0_inverse(code);
    uint32_t q[2] = {0, 0};
    if (code != 0xFFu) {
        const float top = a.e5m2 ? 57344.0f : 448.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __builtin_amdgcn_fmed3f(y[i] * inv, -top, top);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            int p = 0;
            if (a.e5m2) {
                p = __builtin_amdgcn_cvt_pk_bf8_f32(y[4 * g], y[4 * g + 1], p, false);
                p = __builtin_amdgcn_cvt_pk_bf8_f32(y[4 * g + 2], y[4 * g + 3], p, true);
            } else {
                p = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * g], y[4 * g + 1], p, false);
                p = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * g + 2], y[4 * g + 3], p, true);
            }
            q[g] = (uint32_t)p;
        }
    }
    const uint64_t at = row * a.vectors + v;
    Words2<1> out;
    out.w[0] = q[0];
    out.w[1] = q[1];
    *reinterpret_cast<Words2<1> *>(a.codes + 8 * at) = out;
    if ((v & 3u) == 0) a.scales[at / 4] = (uint8_t)code;
}

__device__ __forceinline__ double norm_factor(const NormArgs &a, double s) { return 1.0 / sqrt(s / (double)a.cols + a.eps); }

// sum over the TPR threads of a row
template <int TPR> __device__ __forceinline__ double row_sum(double s, double *part)
{
    s = wave_sum(s);
    if (TPR == 64) return s;
    const uint32_t wave = threadIdx.x / 64;
    if (threadIdx.x % 64 == 0) part[wave] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int w = 0; w < TPR / 64; ++w) s += part[w];
    return s;
}

template <int T, int TW, int NV, int TPR>
__global__ void __launch_bounds__(TPR == 64 ? 256 : TPR) rmsnorm_kernel(const NormArgs a)
{
    constexpr int ROWS = TPR == 64 ? 4 : 1;
    __shared__ double part[TPR / 64];
    const uint64_t row = (uint64_t)blockIdx.x * ROWS + threadIdx.x / TPR;
    if (row >= a.rows) return;                     // a whole wavefront (and with TPR = 64 none waits at a barrier)
    const uint32_t t = threadIdx.x % TPR;
    Raw8<T> h[NV];
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (t + i * TPR < a.vectors) h[i] = norm_input<T>(a, row, t + i * TPR);
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (t + i * TPR < a.vectors) s = squares<T>(h[i], s);
    const double r = norm_factor(a, row_sum<TPR>(s, part));
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (t + i * TPR < a.vectors) norm_output<T, TW>(a, row, t + i * TPR, h[i], r);
}

// Rows longer than a workgroup's registers: two passes, the second on what the first left in the caches.  Where
// residual_out is written it is read back (each thread its own stores: x or the residual may lie in the same memory).
template <int T, int TW>
__global__ void __launch_bounds__(1024) rmsnorm_long_kernel(const NormArgs a)
{
    __shared__ double part[16];
    const uint64_t row = blockIdx.x;
    double s = 0.0;
    for (uint32_t v = threadIdx.x; v < a.vectors; v += 1024) s = squares<T>(norm_input<T>(a, row, v), s);
    const double r = norm_factor(a, row_sum<1024>(s, part));
    NormArgs b = a;
    if (a.residual_out) {
        b.x = a.residual_out;
        b.x_stride = a.residual_stride;
        b.residual = nullptr;
    }
    b.residual_out = nullptr;
    for (uint32_t v = threadIdx.x; v < a.vectors; v += 1024) norm_output<T, TW>(a, row, v, norm_input<T>(b, row, v), r);
}

// Threads of a row and vectors of a thread, by the row's length.  What the choice was measured against, BF16 with a residual, us: 1024 columns, 8192
// rows without one: 10.8 with 64 threads, 12.8 with 256; 4096 columns, 1 and 4096 rows: 4.0 and 29.0 with 512 threads, 4.4 and 29.4 with 256; 8192 columns, 96
// and 8192 rows: 5.1 and 91 with 512 threads, 6.6 and 93 with 256, 5.2 and 97 with 1024.  (512 threads for rows of 2048 columns: 34 against 29.)
template <int T, int TW> static mmaemu_status launch_typed(const NormArgs &a, hipStream_t s)
{
#define MMAEMU_NORM(NV, TPR)                                                                                                         \
    hipLaunchKernelGGL((rmsnorm_kernel<T, TW, NV, TPR>), dim3((uint32_t)(TPR == 64 ? (a.rows + 3) / 4 : a.rows)), dim3(TPR == 64 ? 256 : TPR), 0, s, a)
    const uint32_t v = a.vectors;
    if (v <= 64) MMAEMU_NORM(1, 64);
    else if (v <= 128) MMAEMU_NORM(2, 64);
    else if (v <= 256) MMAEMU_NORM(1, 256);
    else if (v <= 512) MMAEMU_NORM(1, 512);
    else if (v <= 1024) MMAEMU_NORM(2, 512);
    else if (v <= 2048) MMAEMU_NORM(2, 1024);
    else if (v <= 4096) MMAEMU_NORM(4, 1024);
    else hipLaunchKernelGGL((rmsnorm_long_kernel<T, TW>), dim3((uint32_t)a.rows), dim3(1024), 0, s, a);
#undef MMAEMU_NORM
    MMAEMU_HIP(hipGetLastError());
    return MMAEMU_OK;
}

mmaemu_status launch_rmsnorm_quantize(const void *x, const void *residual, const void *weight, void *residual_out, void *codes, void *scales,
                                      uint64_t rows, uint32_t cols, uint64_t x_stride, uint64_t residual_stride, uint32_t type,
                                      uint32_t weight_type, uint32_t code_type, uint32_t scale_rule, double eps, hipStream_t s)
{
    const uint32_t vectors = (cols + 31) / 32 * 4, eb = type == MMAEMU_FP32 ? 4 : 2;
    constexpr uint64_t MOST = 1ull << 21;                              // rows of one launch: its threads count in 32 bits
    for (uint64_t r0 = 0; r0 < rows; r0 += MOST) {
        const uint64_t ro = r0 * residual_stride * eb;
        const NormArgs a = {(const char *)x + r0 * x_stride * eb, residual ? (const char *)residual + ro : nullptr, weight,
                            residual_out ? (char *)residual_out + ro : nullptr, (uint8_t *)codes + r0 * vectors * 8, (uint8_t *)scales + r0 * (vectors / 4),
                            rows - r0 < MOST ? rows - r0 : MOST, x_stride, residual_stride, cols, vectors, code_type == MMAEMU_FP8_E5M2,
                            scale_rule == MMAEMU_SCALE_RULE_FIT, eps};
        const bool wide = weight_type == MMAEMU_FP32;
        mmaemu_status st;
        switch (type) {
        case MMAEMU_BF16: st = wide ? launch_typed<MMAEMU_BF16, MMAEMU_FP32>(a, s) : launch_typed<MMAEMU_BF16, MMAEMU_BF16>(a, s); break;
        case MMAEMU_FP16: st = wide ? launch_typed<MMAEMU_FP16, MMAEMU_FP32>(a, s) : launch_typed<MMAEMU_FP16, MMAEMU_FP16>(a, s); break;
        default: st = launch_typed<MMAEMU_FP32, MMAEMU_FP32>(a, s); break;
        }
        if (st != MMAEMU_OK) return st;
    }
    return MMAEMU_OK;
}

} // namespace mmaemu
