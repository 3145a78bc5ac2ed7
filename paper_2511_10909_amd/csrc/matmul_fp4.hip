// D = alpha A W^T with W in packed FP4 (E2M1) under group scales: MXFP4 (E8M0 per 32 products) or NVFP4 (UE4M3 per 16), and A in
// BF16 or FP16, or in E4M3 / E5M2 with E8M0 scales per 32.
#include "fp4_operands.hpp"

namespace mmaemu {

// Few tokens: the weights are read once, by the wavefront that multiplies them; nothing is shared but the sum.  A workgroup's
// wavefronts take the same 16 tokens x 16 NT weight rows and each a contiguous part of the products; their sums meet in LDS.
//
// Each wavefront keeps a ring of two slots of DW windows in LDS that only it uses: copies by the memory system fill the slots
// ahead, and no barrier is needed.  Loads straight into registers are slower: the instructions want sixteen rows in
// consecutive lanes, and the first-level cache looks up a line for each lane then, 64 for a load; the copies run along the rows.
template <int AT, int SF, int MR, int NT, int DW, int WAVES> struct Stream {
    static constexpr bool BYTES = AT == MMAEMU_FP8_E4M3 || AT == MMAEMU_FP8_E5M2;
    static constexpr int R = 2;                                        // slots (three and four are no faster)
    static constexpr int XB = BYTES ? 128 : 256;                       // bytes of a token per window
    static constexpr int WROW = 64 * DW;                               // bytes of a weight row per slot
    static constexpr int SB = SF == MMAEMU_SCALE_FORMAT_E8M0 ? 4 : 8;  // scale bytes of a weight row per window
    static constexpr int W_BYTES = 16 * NT * WROW, X_BYTES = DW * MR * XB, SLOT = W_BYTES + X_BYTES;
    static constexpr int WC = W_BYTES / 1024, XC = (X_BYTES + 1023) / 1024, COPIES = WC + XC;
    static constexpr int RUN = 64 / SB;                                // windows whose scales are staged together: 64 bytes of a weight row
    static constexpr int SW_ROW = RUN * SB, SX_ROW = RUN * 4;          // bytes of a row's scales in a run,
    static constexpr int SW_PITCH = SW_ROW + 16, SX_PITCH = SX_ROW + 16;               // and what rows are apart: no two in a bank
    static constexpr int SW_BYTES = 16 * NT * SW_PITCH, SX_BYTES = BYTES ? MR * SX_PITCH : 0;
    static constexpr int WAVE_LDS = R * SLOT + SW_BYTES + SX_BYTES;
    static constexpr int SUM_LDS = NT * WAVES * 1024;
    static constexpr int LDS = WAVES * WAVE_LDS > SUM_LDS ? WAVES * WAVE_LDS : SUM_LDS;
};

// one window: weights w with scales s, MT x XW pieces of activations
template <int AT, int SF> __device__ __forceinline__ f32x4 window_products(u32x4 w, uint32_t s, const u32x4 (&x)[AT == MMAEMU_FP8_E4M3 || AT == MMAEMU_FP8_E5M2 ? 2 : 4], uint32_t sx, f32x4 acc)
{
    if constexpr (AT == MMAEMU_FP8_E4M3 || AT == MMAEMU_FP8_E5M2) {
        const i32x8 v = {(int)x[0][0], (int)x[0][1], (int)x[0][2], (int)x[0][3], (int)x[1][0], (int)x[1][1], (int)x[1][2], (int)x[1][3]};
        return mfma_scaled<AT>(w, s, v, sx, acc);
    } else if constexpr (SF == MMAEMU_SCALE_FORMAT_UE4M3) {
        const f16x2 sh = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(s & 0x7F7Fu, 1.0f, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const _Float16 sj = sh[j / 2];
            if constexpr (AT == MMAEMU_FP16) acc = mfma_fp16(weights_fp16_by(w[j], f16x2{sj, sj}), Frag16{x[j]}, acc);
            else acc = mfma_bf16(weights_bf16_by(w[j], (float)sj), Frag16{x[j]}, acc);
        }
    } else if (AT == MMAEMU_BF16 || !__all(fp16_holds(s))) {
        const bool far = AT == MMAEMU_FP16 && any_far(s);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const Frag16 f = weights_second_way(w[j], s, far);
            if (AT == MMAEMU_FP16) {
                Frag16 hi, lo;
                split_fp16(Frag16{x[j]}, far ? 4.0f : 1.0f, hi, lo);
                acc = mfma_bf16(f, lo, acc);
                acc = mfma_bf16(f, hi, acc);
                __builtin_amdgcn_sched_barrier(0);                     // (rare: the parts of one piece at a time in registers)
            } else acc = mfma_bf16(f, Frag16{x[j]}, acc);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) acc = mfma_fp16(weights_fp16(w[j], s), Frag16{x[j]}, acc);
    }
    return acc;
}

template <int AT, int SF, int MR, int NT, int DW, int WAVES> __global__ void __launch_bounds__(64 * WAVES) stream_kernel(const ProductArgs p)
{
    typedef Stream<AT, SF, MR, NT, DW, WAVES> T;
    extern __shared__ __attribute__((aligned(1024))) uint8_t lds[];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, r = lane & 15u;
    const uint32_t n0 = blockIdx.x * (16 * NT);
    uint8_t *const ring = lds + wave * T::WAVE_LDS, *const sw_lds = ring + T::R * T::SLOT, *const sx_lds = sw_lds + T::SW_BYTES;
    // this wavefront's slots of the row
    const uint32_t slots = (p.k + 128 * DW - 1) / (128 * DW), per = slots / WAVES, more = slots % WAVES;
    const uint32_t first = wave * per + (wave < more ? wave : more), count = per + (wave < more ? 1 : 0);

    // sources of this lane's copies, chunks stored where lds_rotation puts them
    const uint8_t *src[T::COPIES];
    uint32_t src_k[T::COPIES];                     // products before the chunk, within the slot
    bool src_in[T::COPIES];
#pragma unroll
    for (int i = 0; i < T::WC; ++i) {
        const uint32_t chunk = 64 * i + lane, row = chunk / (4 * DW), pos = chunk % (4 * DW);
        const uint32_t c = pos ^ lds_rotation<4 * DW>(row);
        const uint32_t n = n0 + row < p.n ? n0 + row : p.n - 1;
        src[i] = p.W + (uint64_t)n * (p.k / 2) + (uint64_t)first * T::WROW + 16 * c;
        src_k[i] = 32 * c;
        src_in[i] = true;
    }
#pragma unroll
    for (int i = 0; i < T::XC; ++i) {
        constexpr uint32_t PER_ROW = T::XB / 16;
        const uint32_t chunk = 64 * i + lane, win = chunk / (MR * PER_ROW), row = chunk / PER_ROW % MR, pos = chunk % PER_ROW;
        const uint32_t c = pos ^ lds_rotation<T::XB / 16>(row);
        const uint32_t m = row;
        src_in[T::WC + i] = chunk < (uint32_t)T::X_BYTES / 16;          // (tokens that are not there: the last one again)
        src[T::WC + i] = p.A + (uint64_t)(m < p.m ? m : p.m - 1) * p.a_stride + (uint64_t)first * (DW * T::XB) + win * T::XB + 16 * c;
        src_k[T::WC + i] = 128 * win + (T::BYTES ? 16 : 8) * c;
    }
    auto issue = [&](uint32_t d) MMAEMU_INLINE {                 // the copies of this wavefront's slot d
        const uint32_t slot = lds_address(ring) + (d % T::R) * T::SLOT;
        if ((first + d + 1) * (128 * DW) > p.k) {
            // the slot that ends inside: zeros first, then what is there
            for (uint32_t c = lane; c < (uint32_t)T::SLOT / 16; c += 64) *reinterpret_cast<u32x4 *>(ring + (d % T::R) * T::SLOT + 16 * c) = u32x4{0, 0, 0, 0};
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
            for (int i = 0; i < T::COPIES; ++i)
                if (src_in[i] && (first + d) * (128 * DW) + src_k[i] < p.k) copy_to_lds(src[i] + (uint64_t)d * (i < T::WC ? T::WROW : DW * T::XB), slot + (i < T::WC ? 1024 * i : T::W_BYTES + 1024 * (i - T::WC)));
            return;
        }
#pragma unroll
        for (int i = 0; i < T::WC; ++i) copy_to_lds(src[i] + (uint64_t)d * T::WROW, slot + 1024 * i);
#pragma unroll
        for (int i = 0; i < T::XC; ++i)
            if (src_in[T::WC + i]) copy_to_lds(src[T::WC + i] + (uint64_t)d * (DW * T::XB), slot + T::W_BYTES + 1024 * i);
    };
    // scales of a run of windows from this wavefront's slot d on: sixteen bytes per lane, byte by byte at a row's end
    auto stage_scales = [&](uint32_t d) MMAEMU_INLINE {
        constexpr uint32_t W_PIECES = 16 * NT * T::SW_ROW / 16, PIECES = W_PIECES + (T::BYTES ? MR * T::SX_ROW / 16 : 0);
        const uint32_t w0 = (first + d) * DW;      // first window
#pragma unroll
        for (uint32_t q0 = 0; q0 < PIECES; q0 += 64) {
            const uint32_t q = q0 + lane;
            if (PIECES % 64 && q >= PIECES) break;
            const bool of_w = q < W_PIECES;
            const uint32_t x = q - W_PIECES, row = of_w ? q / (T::SW_ROW / 16) : x / (T::SX_ROW / 16), at = 16 * (of_w ? q % (T::SW_ROW / 16) : x % (T::SX_ROW / 16));
            const uint32_t n = n0 + row < p.n ? n0 + row : p.n - 1, m = row < p.m ? row : p.m - 1;
            const uint32_t all = of_w ? p.k / (128 / T::SB) : p.k / 32, begin = w0 * (of_w ? T::SB : 4) + at;
            const uint8_t *from = (of_w ? p.SW + (uint64_t)n * all : p.SA + (uint64_t)m * all) + begin;
            Words4<1> v;
            if (begin + 16 <= all) v = *reinterpret_cast<const Words4<1> *>(from);
            else {
#pragma unroll
                for (int e = 0; e < 4; ++e) v.w[e] = SF == MMAEMU_SCALE_FORMAT_UE4M3 ? 0x38383838u : 0x7F7F7F7Fu;
#pragma unroll
                for (uint32_t e = 0; e < 15; ++e)
                    if (begin + e < all) v.w[e / 4] = (v.w[e / 4] & ~(0xFFu << (8 * (e % 4)))) | (uint32_t)from[e] << (8 * (e % 4));
            }
            *reinterpret_cast<u32x4 *>((of_w ? sw_lds + row * T::SW_PITCH : sx_lds + row * T::SX_PITCH) + at) = u32x4{v.w[0], v.w[1], v.w[2], v.w[3]};
        }
    };

    const bool ends_inside = (first + count) * (128 * DW) > p.k;
    f32x4 acc[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[j] = f32x4{0, 0, 0, 0};
    for (uint32_t d = 0; d < T::R && d < count; ++d) issue(d);
    for (uint32_t d = 0; d < count; ++d) {
        if (d % (T::RUN / DW) == 0) stage_scales(d);
        // the next slot may still be under way (one that ends inside counts as none: it may have fewer copies)
        const uint32_t left = count - d - 1;
        if (left > 1 || (left == 1 && !ends_inside)) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(T::COPIES) : "memory");
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        const uint8_t *slot = ring + (d % T::R) * T::SLOT, *xs = slot + T::W_BYTES;
        const uint32_t rx = r % MR;
#pragma unroll
        for (int h = 0; h < DW; ++h) {
            const uint32_t win = d % (T::RUN / DW) * DW + h;
            u32x4 x[T::BYTES ? 2 : 4];
            uint32_t sx = 0;
            if constexpr (T::BYTES) {
                const uint8_t *row = xs + (h * MR + rx) * 128;
                const uint32_t rot = lds_rotation<8>(rx);
                x[0] = *reinterpret_cast<const u32x4 *>(row + 16 * (g ^ rot));
                x[1] = *reinterpret_cast<const u32x4 *>(row + 16 * ((4 + g) ^ rot));
                sx = sx_lds[rx * T::SX_PITCH + 4 * win + g];
            } else {
                const uint8_t *row = xs + (h * MR + rx) * 256;
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = *reinterpret_cast<const u32x4 *>(row + 16 * ((4 * g + j) ^ lds_rotation<16>(rx)));
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const uint32_t c = (4 * h + g) ^ lds_rotation<4 * DW>(r);
                const u32x4 w = *reinterpret_cast<const u32x4 *>(slot + (16 * j + r) * T::WROW + 16 * c);
                const uint8_t *sr = sw_lds + (16 * j + r) * T::SW_PITCH + T::SB * win;
                const uint32_t sc = SF == MMAEMU_SCALE_FORMAT_E8M0 ? sr[g] : *reinterpret_cast<const uint16_t *>(sr + 2 * g);
                acc[j] = window_products<AT, SF>(w, sc, x, sx, acc[j]);
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");             // everything of the slot has been read
        if (d + T::R < count) issue(d + T::R);
    }
    __syncthreads();
    f32x4 *part = reinterpret_cast<f32x4 *>(lds);
#pragma unroll
    for (int j = 0; j < NT; ++j) part[(j * WAVES + wave) * 64 + lane] = acc[j];
    __syncthreads();
    for (uint32_t t = wave; t < NT; t += WAVES) {
        f32x4 sum = part[t * WAVES * 64 + lane];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) sum += part[(t * WAVES + w) * 64 + lane];
        with_output_type(p.d_type, [&](auto dt) { store_outputs<dt.value>(p, r, n0 + 16 * t + 4 * g, sum); });
    }
}

template <int AT, int SF, int MR, int NT, int DW, int WAVES> static mmaemu_status launch_stream(const ProductArgs &p, hipStream_t s)
{
    typedef Stream<AT, SF, MR, NT, DW, WAVES> T;
    static_assert(T::LDS <= 160 * 1024, "ring");
    hipLaunchKernelGGL((stream_kernel<AT, SF, MR, NT, DW, WAVES>), dim3((p.n + 16 * NT - 1) / (16 * NT)), dim3(64 * WAVES), T::LDS, s, p);
    MMAEMU_HIP(hipGetLastError());
    return MMAEMU_OK;
}

// Up to sixteen tokens go through the stream (32 x 32 blocks take 13 us against 10.5 for 16 BF16 tokens on 8192 x 8192 MXFP4 weights, 11
// against 8.9 for E4M3 ones; at 32 tokens the stream reads the weights twice).
constexpr uint32_t STREAM_TOKENS = 16;

// Rows of a slot's activations (MR): those that the tokens fill, 4, 8 or 16; fewer cost less of the copies' rate (one BF16 token on
// 28672 x 8192: 24 us with 4 rows, 37 with 16; 7 E4M3 tokens, 7552 x 3904: 8.5 with 16 rows, 7.4 with 8).
// Wavefronts: eight instead of four up to 4096 weight rows, where few workgroups share long rows (one BF16 token, 1024 x 16384: 7.0 -> 5.9 us).
// Windows of a slot (DW): two; four where rows are no whole lines of 128 bytes, as long as all workgroups are resident with them (one E4M3
// token, 3633 x 4288: 5.8 -> 4.8, 7552 x 3904: 7.1 -> 6.6; but 13824 x 3776: 8.5 -> 10.6).
// Weight rows of a workgroup (16 NT): 16 until the activations, which every workgroup reads, cost more than idle units, and one window a
// slot where that is what lets all workgroups be resident.  16-bit activations, us (E8M0 and UE4M3 scales):
//   7 tokens, 8192 x 8192: 16 rows x 2 windows 7.8 and 8.7, 32 x 2 8.1 and 10.0;  13824 x 3776: 16 x 2 12.1 and 13.1, 16 x 1 10.3 and 10.3,
//     32 x 2 10.3 and 11.4;  20000 x 5120: 16 x 1 14.0 and 13.7, 32 x 2 18.7 and 16.2;  12864 x 8192: 16 x 1 13.2 and 15.1, 32 x 2 11.5 and 13.5
//   14 tokens, 7552 x 3904: 16 x 1 8.6 and 8.1, 32 x 1 9.3 and 9.1;  8192 x 8192: 32 x 2 9.1 and 11.0, 32 x 1 9.8 and 10.7, 32 x 1 of eight
//     wavefronts 10.3 and 10.2;  13824 x 3776: 32 x 1 12.1 and 11.7, 64 x 1 14.0 and 14.4
// 8-bit ones: 14 tokens, 7552 x 3904: 16 x 2 7.9, 32 x 2 8.6;  13824 x 3776: 12.9 and 10.1
// Beyond 8192 weight rows: fifteen numbers of them up to 131072, rows of 1024 to 16384 products, 6 to 16 tokens.  The time of what is taken, over that
// of the fastest of these shapes: 1.02 to 1.07 in the mean of a kind and number of tokens, at most 1.42 (8-bit, 20480 x 1024).  On either side of the limits, us:
//   16-bit, 8 tokens, BF16 on E8M0: 40960 x 2048: 16 x 1 10.8, 32 x 2 14.2;  57344 x 4096: 34.1 and 29.8;  20480 x 6144 (FP16): 14.4 and 18.2;  14336 x 8192
//     (FP16) and longer rows: 32 x 2
//   16-bit, 14 tokens: 20480 x 4096: 16 x 1 13.1, 32 x 1 13.4, 64 x 1 17.4;  24576 x 8192: 16 x 1 a fifth slower than 32 x 1;  28672 x 4096 18.5 with 64 x 1, 16.1 with
//     32 x 1;  131072 x 2048 55 and 45;  128256 x 8192 134 and 142, but on UE4M3 193 and 171
//   8-bit, 14 tokens: 20000 x 5120: 32 x 2 18.4, 32 x 1 14.2;  28672 x 8192: 27 and 31;  131072 x 2048: 41 and 35
template <int AT, int SF> static mmaemu_status launch_stream_typed(const ProductArgs &p, hipStream_t s)
{
    constexpr bool BYTES = AT == MMAEMU_FP8_E4M3 || AT == MMAEMU_FP8_E5M2, E8M0 = SF == MMAEMU_SCALE_FORMAT_E8M0;
    const bool few = p.n <= 4096, resident = p.n <= 8192, ragged = p.k % 256 != 0;
    if (p.m <= 4) {
        if (few) return ragged ? launch_stream<AT, SF, 4, 1, 4, 8>(p, s) : launch_stream<AT, SF, 4, 1, 2, 8>(p, s);
        return resident && ragged ? launch_stream<AT, SF, 4, 1, 4, 4>(p, s) : launch_stream<AT, SF, 4, 1, 2, 4>(p, s);
    }
    if constexpr (BYTES) {
        if (p.m <= 8) {
            if (few) return ragged ? launch_stream<AT, SF, 8, 1, 4, 8>(p, s) : launch_stream<AT, SF, 8, 1, 2, 8>(p, s);
            return resident && ragged ? launch_stream<AT, SF, 8, 1, 4, 4>(p, s) : launch_stream<AT, SF, 8, 1, 2, 4>(p, s);
        }
        if (few) return launch_stream<AT, SF, 16, 1, 2, 8>(p, s);
        if (resident) return launch_stream<AT, SF, 16, 1, 2, 4>(p, s);
        return p.n > 16384 && p.k <= (p.n <= 24576 ? 6144 : 2048) ? launch_stream<AT, SF, 16, 2, 1, 4>(p, s) : launch_stream<AT, SF, 16, 2, 2, 4>(p, s);
    } else {
        if (p.m <= 8) {
            if (few) return launch_stream<AT, SF, 8, 1, 2, 8>(p, s);
            if (resident) return launch_stream<AT, SF, 8, 1, 2, 4>(p, s);
            return p.k <= (p.n <= 20480 ? 6144 : 2048) ? launch_stream<AT, SF, 8, 1, 1, 4>(p, s) : launch_stream<AT, SF, 8, 2, 2, 4>(p, s);
        }
        if (few) return launch_stream<AT, SF, 16, 1, 1, 8>(p, s);
        if (resident && p.k <= 4096) return launch_stream<AT, SF, 16, 1, 1, 4>(p, s);
        if (resident) {
            if constexpr (E8M0) return launch_stream<AT, SF, 16, 2, 2, 4>(p, s);
            else return launch_stream<AT, SF, 16, 2, 1, 8>(p, s);
        }
        if (p.n > 16384 && p.n <= 24576 && p.k <= 6144) return launch_stream<AT, SF, 16, 1, 1, 4>(p, s);
        if constexpr (E8M0)
            if (p.n > 24576 && p.k > 6144) return launch_stream<AT, SF, 16, 4, 1, 4>(p, s);
        return launch_stream<AT, SF, 16, 2, 1, 4>(p, s);
    }
}

mmaemu_status launch_matmul_fp4(const void *A, const void *SA, const void *W, const void *SW, void *D, uint32_t m, uint32_t n, uint32_t k,
                                uint64_t a_stride, uint64_t d_stride, uint32_t a_type, uint32_t d_type, uint32_t scale_format, float alpha, hipStream_t s)
{
    const bool bytes = is_byte_type(a_type), e8m0 = scale_format == MMAEMU_SCALE_FORMAT_E8M0;
    const ProductArgs p = {(const uint8_t *)A, (const uint8_t *)SA, (const uint8_t *)W, (const uint8_t *)SW, D, a_stride * (bytes ? 1 : 2), d_stride, m, n, k,
                           d_type, alpha};
    if (m > STREAM_TOKENS) return launch_tiled(p, a_type, scale_format, s);
    switch (a_type) {
    case MMAEMU_FP8_E4M3: return launch_stream_typed<MMAEMU_FP8_E4M3, MMAEMU_SCALE_FORMAT_E8M0>(p, s);
    case MMAEMU_FP8_E5M2: return launch_stream_typed<MMAEMU_FP8_E5M2, MMAEMU_SCALE_FORMAT_E8M0>(p, s);
    case MMAEMU_BF16: return e8m0 ? launch_stream_typed<MMAEMU_BF16, MMAEMU_SCALE_FORMAT_E8M0>(p, s) : launch_stream_typed<MMAEMU_BF16, MMAEMU_SCALE_FORMAT_UE4M3>(p, s);
    default: return e8m0 ? launch_stream_typed<MMAEMU_FP16, MMAEMU_SCALE_FORMAT_E8M0>(p, s) : launch_stream_typed<MMAEMU_FP16, MMAEMU_SCALE_FORMAT_UE4M3>(p, s);
    }
}

const char *matmul_fp4_kernel_name(uint32_t m, uint32_t n, uint32_t k, uint32_t a_type, uint32_t scale_format)
{
    return m > STREAM_TOKENS ? tiled_name(m, n, k, a_type, scale_format) : "stream";
}

} // namespace mmaemu
