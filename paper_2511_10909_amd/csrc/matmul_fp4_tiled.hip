// Products with packed FP4 weights for many rows: tiles of BM tokens x BN weight rows per workgroup, both operands staged through
// LDS by the memory system's own copies, three buffers deep.
#include "fp4_operands.hpp"

namespace mmaemu {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// One step is 128 bytes of an activation row: 128 products of 8-bit activations, 64 of 16-bit ones.  Scales are staged for
// sixteen bytes of a row at a time (GROUP steps).
template <int AT, int SF, int BM, int BN, int TM, int TN> struct Tile {
    static constexpr bool BYTES = AT == MMAEMU_FP8_E4M3 || AT == MMAEMU_FP8_E5M2;
    static constexpr int KS = BYTES ? 128 : 64;                        // products per step
    static constexpr int WB = KS / 2;                                  // bytes of a weight row
    static constexpr int PER_SCALE = SF == MMAEMU_SCALE_FORMAT_E8M0 ? 32 : 16;
    static constexpr int SB = KS / PER_SCALE;                          // scale bytes of a row
    static constexpr int GROUP = 16 / SB;
    static constexpr int THREADS = 64 * (BM / TM) * (BN / TN);
    static constexpr int A_BYTES = BM * 128, W_BYTES = BN * WB, STAGE = A_BYTES + W_BYTES;
    static constexpr int STAGES = 3;
    static constexpr int SCALE_ROWS = (BYTES ? BM : 0) + BN;           // of activations, then of weights
    static constexpr int SCALES = SCALE_ROWS * 16;
    static constexpr int LDS = STAGES * STAGE + 2 * SCALES;
    static constexpr int COPIES = STAGE / (16 * THREADS);              // of 16 bytes, per thread and step
    static constexpr int SPER = (SCALE_ROWS + THREADS - 1) / THREADS;
};

__device__ __forceinline__ uint32_t lds_address(const uint8_t *p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) uint8_t *)p; }

// Sixteen bytes per lane from memory to LDS, to + 16 lane.  By hand: before a read the compiler waits for every copy that it
// knows of, as it cannot tell the buffers apart.  No register is written, and the address is read as the copy is issued.
__device__ __forceinline__ void copy_to_lds(const uint8_t *from, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(to) : "memory");
}

template <int AT, int SF, int BM, int BN, int TM, int TN>
__global__ void __launch_bounds__((Tile<AT, SF, BM, BN, TM, TN>::THREADS)) tiled_kernel(const ProductArgs p, uint32_t tiles_m, uint32_t tiles_n)
{
    typedef Tile<AT, SF, BM, BN, TM, TN> T;
    extern __shared__ __attribute__((aligned(256))) uint8_t lds[];
    uint8_t *const scales = lds + T::STAGES * T::STAGE;
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, r = lane & 15u;
    // workgroups go round the eight dies: each die takes a contiguous run of tiles, in columns of eight token tiles
    const uint32_t total = tiles_m * tiles_n, id = blockIdx.x;
    const uint32_t per = total / 8, more = total % 8, die = id % 8;
    const uint32_t t = die * per + (die < more ? die : more) + id / 8;
    const uint32_t band = 8 * tiles_n, b = t / band, inb = t - b * band, high = tiles_m - 8 * b < 8 ? tiles_m - 8 * b : 8;
    const uint32_t m0 = (8 * b + inb % high) * BM, n0 = (inb / high) * BN;
    const uint32_t full = p.k / T::KS, steps = (p.k + T::KS - 1) / T::KS, row_scales = p.k / T::PER_SCALE;

    // Source of each of this thread's copies: 16-byte chunk c of a row.  Chunks are stored rotated by the row, so that the
    // sixteen rows that lanes read together lie in different banks.
    const uint8_t *src[T::COPIES];
#pragma unroll
    for (int i = 0; i < T::COPIES; ++i) {
        const uint32_t chunk = i * T::THREADS + tid;                   // all of A, then all of W: the same side for all lanes
        if (i * T::THREADS < T::A_BYTES / 16) {
            const uint32_t row = chunk / 8, c = (chunk % 8) ^ ((row >> 1) & 7);
            const uint32_t m = m0 + row < p.m ? m0 + row : p.m - 1;
            src[i] = p.A + (uint64_t)m * p.a_stride + 16 * c;
        } else {
            const uint32_t cw = chunk - T::A_BYTES / 16, row = cw / (T::WB / 16);
            const uint32_t c = T::BYTES ? (cw % 4) ^ ((row >> 2) & 3) : cw % 2;
            const uint32_t n = n0 + row < p.n ? n0 + row : p.n - 1;
            src[i] = p.W + (uint64_t)n * (p.k / 2) + 16 * c;
        }
    }
    auto issue = [&](uint32_t s) {                                     // the copies of a whole step
        const uint32_t to = lds_address(lds) + (s % T::STAGES) * T::STAGE + 1024 * wave;
#pragma unroll
        for (int i = 0; i < T::COPIES; ++i) copy_to_lds(src[i] + (uint64_t)s * (i * T::THREADS < T::A_BYTES / 16 ? 128 : T::WB), to + 16 * i * T::THREADS);
    };

    // scales: row q of the staged ones, sixteen bytes at a time; beyond the row 2^0 (which meets zeros)
    const uint8_t *ssrc[T::SPER];
#pragma unroll
    for (int i = 0; i < T::SPER; ++i) {
        const uint32_t q = i * T::THREADS + tid;
        if (T::BYTES && q < BM) {
            const uint32_t m = m0 + q < p.m ? m0 + q : p.m - 1;
            ssrc[i] = p.SA + (uint64_t)m * row_scales;
        } else {
            const uint32_t row = q - (T::BYTES ? BM : 0), n = n0 + row < p.n ? n0 + row : p.n - 1;
            ssrc[i] = p.SW + (uint64_t)n * row_scales;
        }
    }
    Words4<1> sreg[T::SPER];
    auto load_scales = [&](uint32_t group) {
#pragma unroll
        for (int i = 0; i < T::SPER; ++i) {
            if (16 * group + 16 <= row_scales) {
                sreg[i] = *reinterpret_cast<const Words4<1> *>(ssrc[i] + 16 * group);
                continue;
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) sreg[i].w[e] = SF == MMAEMU_SCALE_FORMAT_UE4M3 ? 0x38383838u : 0x7F7F7F7Fu;
#pragma unroll
            for (uint32_t e = 0; e < 15; ++e)
                if (16 * group + e < row_scales) sreg[i].w[e / 4] = (sreg[i].w[e / 4] & ~(0xFFu << (8 * (e % 4)))) | (uint32_t)ssrc[i][16 * group + e] << (8 * (e % 4));
        }
    };
    auto put_scales = [&](uint32_t group) {
        uint8_t *to = scales + (group & 1) * T::SCALES;
#pragma unroll
        for (int i = 0; i < T::SPER; ++i) {
            const uint32_t q = i * T::THREADS + tid;
            if (T::SCALE_ROWS % T::THREADS != 0 && q >= (uint32_t)T::SCALE_ROWS) continue;
            *reinterpret_cast<u32x4 *>(to + 16 * q) = u32x4{sreg[i].w[0], sreg[i].w[1], sreg[i].w[2], sreg[i].w[3]};
        }
    };

    constexpr int MT = TM / 16, NT = TN / 16;
    const uint32_t wm = (wave % (BM / TM)) * TM, wn = (wave / (BM / TM)) * TN;
    const uint32_t rot = (r >> 1) & 7;                                 // (tiles begin at multiples of 16 rows)
    f32x4 acc[NT][MT];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[j][i] = f32x4{0, 0, 0, 0};

    auto compute = [&](uint32_t s) {
        const uint8_t *a = lds + (s % T::STAGES) * T::STAGE + (wm + r) * 128, *w = lds + (s % T::STAGES) * T::STAGE + T::A_BYTES + (wn + r) * T::WB;
        const uint8_t *sw = scales + ((s / T::GROUP) & 1) * T::SCALES + (s % T::GROUP) * T::SB, *sa = sw + (wm + r) * 16;
        sw += ((T::BYTES ? BM : 0) + wn + r) * 16;
        if constexpr (T::BYTES) {
            const uint8_t *wl = w + 16 * (g ^ (r >> 2)), *lo = a + 16 * (g ^ rot), *hi = a + 16 * ((4 + g) ^ rot);
            sw += g;
            sa += g;
            u32x4 wf[NT];
            uint32_t ws[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                wf[j] = *reinterpret_cast<const u32x4 *>(wl + 16 * 64 * j);
                ws[j] = sw[256 * j];
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const u32x4 l = *reinterpret_cast<const u32x4 *>(lo + 2048 * i), h = *reinterpret_cast<const u32x4 *>(hi + 2048 * i);
                const i32x8 x = {(int)l[0], (int)l[1], (int)l[2], (int)l[3], (int)h[0], (int)h[1], (int)h[2], (int)h[3]};
                const uint32_t xs = sa[256 * i];
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[j][i] = mfma_scaled<AT>(wf[j], ws[j], x, xs, acc[j][i]);
            }
        } else {
            Frag16 x[2][MT];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h) x[h][i].w = *reinterpret_cast<const u32x4 *>(a + 16 * ((2 * g + h) ^ rot) + 2048 * i);
            const uint8_t *wl = w + 8 * g;
            sw += SF == MMAEMU_SCALE_FORMAT_E8M0 ? g / 2 : g;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const u32x2 c = *reinterpret_cast<const u32x2 *>(wl + 16 * 32 * j);
                const uint32_t s = SF == MMAEMU_SCALE_FORMAT_E8M0 ? sw[256 * j] : sw[256 * j] & 0x7Fu;
                if constexpr (SF == MMAEMU_SCALE_FORMAT_UE4M3) {
                    const f16x2 sh = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(s, 1.0f, 0);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if constexpr (AT == MMAEMU_FP16) {
                            const Frag16 f = weights_fp16_by(c[h], f16x2{sh[0], sh[0]});
#pragma unroll
                            for (int i = 0; i < MT; ++i) acc[j][i] = mfma_fp16(f, x[h][i], acc[j][i]);
                        } else {
                            const Frag16 f = weights_bf16_by(c[h], (float)sh[0]);
#pragma unroll
                            for (int i = 0; i < MT; ++i) acc[j][i] = mfma_bf16(f, x[h][i], acc[j][i]);
                        }
                    }
                } else if constexpr (AT == MMAEMU_BF16) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const Frag16 f = weights_bf16(c[h], s);
#pragma unroll
                        for (int i = 0; i < MT; ++i) acc[j][i] = mfma_bf16(f, x[h][i], acc[j][i]);
                    }
                } else if (__all(fp16_holds(s))) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const Frag16 f = weights_fp16(c[h], s);
#pragma unroll
                        for (int i = 0; i < MT; ++i) acc[j][i] = mfma_fp16(f, x[h][i], acc[j][i]);
                    }
                } else {
                    const bool far = s - 253u < 2u;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const Frag16 f = weights_bf16(c[h], far ? s - 2 : s);
#pragma unroll
                        for (int i = 0; i < MT; ++i) {
                            Frag16 hi, lo;
                            split_fp16(x[h][i], far ? 4.0f : 1.0f, hi, lo);
                            acc[j][i] = mfma_bf16(f, lo, acc[j][i]);
                            acc[j][i] = mfma_bf16(f, hi, acc[j][i]);
                        }
                    }
                }
            }
        }
    };

    // Step s works on its buffer while the copies of step s + 1 come in, and issues those of step s + 2 into the buffer that all
    // wavefronts left before the barrier.  The scales of a group are loaded in the group before and stored in its last step.
    load_scales(0);
    if (full) issue(0);
    put_scales(0);
    if (full > 1) issue(1);
    for (uint32_t s = 0; s < steps; ++s) {
        if (s % T::GROUP == T::GROUP - 1 && s + 1 < steps) put_scales(s / T::GROUP + 1);
        if (s + 1 < full) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(T::COPIES) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (s == full) {                                               // the step that ends inside: products beyond the row are zero times zero
#pragma unroll
            for (int i = 0; i < T::COPIES; ++i) {
                const bool of_a = i * T::THREADS < T::A_BYTES / 16;
                const uint32_t chunk = i * T::THREADS + tid, cw = chunk - T::A_BYTES / 16;
                const uint32_t c = of_a ? (chunk % 8) ^ ((chunk / 16) & 7) : T::BYTES ? (cw % 4) ^ ((cw / 16) & 3) : cw % 2;
                u32x4 v = {0, 0, 0, 0};
                if (s * T::KS + c * (of_a && !T::BYTES ? 8 : of_a ? 16 : 32) < p.k) v = *reinterpret_cast<const u32x4 *>(src[i] + (uint64_t)s * (of_a ? 128 : T::WB));
                *reinterpret_cast<u32x4 *>(lds + (s % T::STAGES) * T::STAGE + 16 * chunk) = v;
            }
            __syncthreads();
        }
        if (s % T::GROUP == 0 && s + T::GROUP < steps) load_scales(s / T::GROUP + 1);
        if (s + 2 < full) issue(s + 2);
        compute(s);
    }
    with_output_type(p.d_type, [&](auto dt) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < MT; ++i) store_outputs<dt.value>(p, m0 + wm + 16 * i + r, n0 + wn + 16 * j + 4 * g, acc[j][i]);
    });
}

template <int AT, int SF, int BM, int BN, int TM, int TN> static mmaemu_status launch_tile(const ProductArgs &p, hipStream_t s)
{
    typedef Tile<AT, SF, BM, BN, TM, TN> T;
    const uint32_t tm = (p.m + BM - 1) / BM, tn = (p.n + BN - 1) / BN;
    static_assert(T::LDS <= 160 * 1024 && (T::A_BYTES / 16) % T::THREADS == 0 && (T::W_BYTES / 16) % T::THREADS == 0, "tile");
    hipLaunchKernelGGL((tiled_kernel<AT, SF, BM, BN, TM, TN>), dim3(tm * tn), dim3(T::THREADS), T::LDS, s, p, tm, tn);
    MMAEMU_HIP(hipGetLastError());
    return MMAEMU_OK;
}

template <int AT, int SF> static mmaemu_status launch_tiled_typed(const ProductArgs &p, hipStream_t s)
{
    return launch_tile<AT, SF, 256, 256, 64, 128>(p, s);
}

mmaemu_status launch_tiled(const ProductArgs &p, uint32_t a_type, uint32_t scale_format, hipStream_t s)
{
    const bool e8m0 = scale_format == MMAEMU_SCALE_FORMAT_E8M0;
    switch (a_type) {
    case MMAEMU_FP8_E4M3: return launch_tiled_typed<MMAEMU_FP8_E4M3, MMAEMU_SCALE_FORMAT_E8M0>(p, s);
    case MMAEMU_FP8_E5M2: return launch_tiled_typed<MMAEMU_FP8_E5M2, MMAEMU_SCALE_FORMAT_E8M0>(p, s);
    case MMAEMU_BF16: return e8m0 ? launch_tiled_typed<MMAEMU_BF16, MMAEMU_SCALE_FORMAT_E8M0>(p, s) : launch_tiled_typed<MMAEMU_BF16, MMAEMU_SCALE_FORMAT_UE4M3>(p, s);
    default: return e8m0 ? launch_tiled_typed<MMAEMU_FP16, MMAEMU_SCALE_FORMAT_E8M0>(p, s) : launch_tiled_typed<MMAEMU_FP16, MMAEMU_SCALE_FORMAT_UE4M3>(p, s);
    }
}

} // namespace mmaemu
