// Products with packed FP4 weights for many rows: tiles of BM tokens x BN weight rows per workgroup, both operands staged through
// LDS by the memory system's own copies, three buffers deep.
#include "fp4_operands.hpp"

namespace mmaemu {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// A part is 128 bytes of an activation row: 128 products of 8-bit activations, 64 of 16-bit ones.  A step is WK parts, one for
// each of the WK wavefronts that share a block of TM x TN outputs; S steps have buffers.
template <int AT, int SF, int BM, int BN, int TM, int TN, int WK, int S> struct Tile {
    static constexpr bool BYTES = AT == MMAEMU_FP8_E4M3 || AT == MMAEMU_FP8_E5M2;
    static constexpr int PART = BYTES ? 128 : 64, KS = PART * WK;      // products
    static constexpr int WB = PART / 2;                                // bytes of a weight row in a part
    static constexpr int PER_SCALE = SF == MMAEMU_SCALE_FORMAT_E8M0 ? 32 : 16;
    static constexpr int SB = PART / PER_SCALE;                        // scale bytes of a row in a part
    static constexpr int GB = SB * WK < 16 ? 16 : SB * WK, GROUP = GB / (SB * WK);     // scale bytes of a row staged together, and their steps
    static constexpr bool IN_REGISTERS = GROUP >= 4;                   // staged through registers (else by copies, as aligned words)
    static constexpr int WPR = IN_REGISTERS ? GB / 4 : GB / 4 + 1;     // words of a row's scales in LDS
    static constexpr int BLOCKS_M = BM / TM, BLOCKS = BLOCKS_M * (BN / TN), THREADS = 64 * BLOCKS * WK;
    static constexpr int A_PART = BM * 128, W_PART = BN * WB, A_BYTES = A_PART * WK, W_BYTES = W_PART * WK, STAGE = A_BYTES + W_BYTES;
    static constexpr int SCALE_ROWS = (BYTES ? BM : 0) + BN;           // of activations, then of weights
    static constexpr int WORDS = SCALE_ROWS * WPR, SCALES = WORDS * 4;
    static constexpr int SUMS = (WK - 1) * BLOCKS * TM * TN * 4;
    static constexpr int LDS = S * STAGE + 2 * SCALES > SUMS ? S * STAGE + 2 * SCALES : SUMS;
    // copies of 16 bytes per thread and step; all wavefronts issue equally many (where there is less to copy than threads, some
    // copy the same twice), as each counts its own
    static constexpr int AC = (A_BYTES / 16 + THREADS - 1) / THREADS, WC = (W_BYTES / 16 + THREADS - 1) / THREADS, COPIES = AC + WC;
};

template <int AT, int SF, int BM, int BN, int TM, int TN, int WK, int S, bool PIPE>
__global__ void __launch_bounds__((Tile<AT, SF, BM, BN, TM, TN, WK, S>::THREADS)) tiled_kernel(const ProductArgs p, uint32_t tiles_m, uint32_t tiles_n)
{
    typedef Tile<AT, SF, BM, BN, TM, TN, WK, S> T;
    extern __shared__ __attribute__((aligned(256))) uint8_t lds[];
    uint8_t *const scales = lds + S * T::STAGE;
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, r = lane & 15u;
    // workgroups go round the eight dies: each die takes a contiguous run of tiles, in columns of eight token tiles
    const uint32_t total = tiles_m * tiles_n, id = blockIdx.x;
    const uint32_t per = total / 8, more = total % 8, die = id % 8;
    const uint32_t t = die * per + (die < more ? die : more) + id / 8;
    const uint32_t band = 8 * tiles_n, b = t / band, inb = t - b * band, high = tiles_m - 8 * b < 8 ? tiles_m - 8 * b : 8;
    const uint32_t m0 = (8 * b + inb % high) * BM, n0 = (inb / high) * BN;
    const uint32_t full = p.k / T::KS, steps = (p.k + T::KS - 1) / T::KS, row_scales = p.k / T::PER_SCALE;

    // Source of each of this thread's copies: part u, row, 16-byte chunk c of it.  Chunks are stored rotated by the row, so that
    // the sixteen rows that lanes read together lie in different banks.
    const uint8_t *src[T::COPIES];
    auto chunk_of = [&](int i) -> uint32_t { return i < T::AC ? (i * T::THREADS + tid) % (T::A_BYTES / 16) : ((i - T::AC) * T::THREADS + tid) % (T::W_BYTES / 16); };
    auto product_of = [&](int i) -> uint32_t {                         // the chunk's first product within the step
        const uint32_t q = chunk_of(i);
        if (i < T::AC) return T::PART * (q / (T::A_PART / 16)) + (T::BYTES ? 16 : 8) * ((q % 8) ^ ((q / 16) & 7));
        return T::PART * (q / (T::W_PART / 16)) + 32 * (T::BYTES ? (q % 4) ^ ((q / 16) & 3) : q % 2);
    };
#pragma unroll
    for (int i = 0; i < T::COPIES; ++i) {
        if (i < T::AC) {
            const uint32_t m = m0 + chunk_of(i) % (T::A_PART / 16) / 8;
            src[i] = p.A + (uint64_t)(m < p.m ? m : p.m - 1) * p.a_stride + product_of(i) * (T::BYTES ? 1 : 2);
        } else {
            const uint32_t n = n0 + chunk_of(i) % (T::W_PART / 16) / (T::WB / 16);
            src[i] = p.W + (uint64_t)(n < p.n ? n : p.n - 1) * (p.k / 2) + product_of(i) / 2;
        }
    }
    auto issue = [&](uint32_t s) {                                     // the copies of a whole step
        const uint32_t to = lds_address(lds) + (s % S) * T::STAGE;
#pragma unroll
        for (int i = 0; i < T::COPIES; ++i) {
            const uint32_t q = i < T::AC ? (i * T::THREADS + 64 * wave) % (T::A_BYTES / 16) : T::A_BYTES / 16 + ((i - T::AC) * T::THREADS + 64 * wave) % (T::W_BYTES / 16);
            copy_to_lds(src[i] + (uint64_t)s * (i < T::AC ? 128 * WK : T::WB * WK), to + 16 * q);
        }
    };

    // Scales, GB bytes of a row at a time.  Where that is four steps and more, a thread loads a row's into registers in the group
    // before and stores them at the barrier before the group; the compiler then waits for the copies under way as well, which costs less
    // than the instructions of the other way (8192^3, E4M3: 438 against 477 us).  Where it is fewer, copies bring the aligned
    // words that hold them (a row begins at any byte; reads are of bytes).  Bytes beyond a row are 2^0 (they meet zeros).
    auto scale_row = [&](uint32_t q) -> const uint8_t * {              // of activations, then of weights
        if (T::BYTES && q < (uint32_t)BM) return p.SA + (uint64_t)(m0 + q < p.m ? m0 + q : p.m - 1) * row_scales;
        const uint32_t n = n0 + q - (T::BYTES ? BM : 0);
        return p.SW + (uint64_t)(n < p.n ? n : p.n - 1) * row_scales;
    };
    constexpr uint32_t ONES = SF == MMAEMU_SCALE_FORMAT_UE4M3 ? 0x38383838u : 0x7F7F7F7Fu;
    constexpr int REGS = T::IN_REGISTERS ? (T::SCALE_ROWS + T::THREADS - 1) / T::THREADS : 1;
    Words4<1> sreg[REGS];
    auto load_scales = [&](uint32_t group) {
#pragma unroll
        for (int i = 0; i < REGS; ++i) {
            const uint32_t q = i * T::THREADS + tid;
            const uint8_t *from = scale_row(q < (uint32_t)T::SCALE_ROWS ? q : 0) + 16 * group;
            if (16 * group + 16 <= row_scales) sreg[i] = *reinterpret_cast<const Words4<1> *>(from);
            else {
#pragma unroll
                for (int e = 0; e < 4; ++e) sreg[i].w[e] = ONES;
#pragma unroll
                for (uint32_t e = 0; e < 15; ++e)
                    if (16 * group + e < row_scales) sreg[i].w[e / 4] = (sreg[i].w[e / 4] & ~(0xFFu << (8 * (e % 4)))) | (uint32_t)from[e] << (8 * (e % 4));
            }
        }
    };
    auto word_of = [&](uint32_t q, uint32_t group) -> const uint8_t * {
        const uint8_t *from = scale_row(q / T::WPR) + T::GB * group;
        return from - ((uintptr_t)from & 3) + 4 * (q % T::WPR);
    };
    auto put_scales = [&](uint32_t group) {
        uint8_t *to = scales + (group & 1) * T::SCALES;
        if constexpr (T::IN_REGISTERS) {
#pragma unroll
            for (int i = 0; i < REGS; ++i) {
                const uint32_t q = i * T::THREADS + tid;
                if (T::SCALE_ROWS % T::THREADS == 0 || q < (uint32_t)T::SCALE_ROWS) *reinterpret_cast<u32x4 *>(to + 16 * q) = u32x4{sreg[i].w[0], sreg[i].w[1], sreg[i].w[2], sreg[i].w[3]};
            }
        } else {
            for (uint32_t q = tid; q < (uint32_t)T::WORDS; q += T::THREADS) {
                const uint8_t *begin = scale_row(q / T::WPR), *end = begin + row_scales, *from = word_of(q, group);
                uint32_t w = ONES;
                if (from >= begin && from + 4 <= end) w = *reinterpret_cast<const uint32_t *>(from);
                else
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (from + e >= begin && from + e < end) w = (w & ~(0xFFu << (8 * e))) | (uint32_t)from[e] << (8 * e);
                *reinterpret_cast<uint32_t *>(to + 4 * q) = w;
            }
        }
    };
    // copies do it where all words lie within their rows (with rows of aligned words the last is not needed)
    const bool words = row_scales % 4 == 0 && ((uintptr_t)p.SW & 3) == 0 && (!T::BYTES || ((uintptr_t)p.SA & 3) == 0);
    auto copies_do = [&](uint32_t group) { return !T::IN_REGISTERS && T::GB * group + (words ? T::GB : T::GB + 4) <= row_scales; };
    auto copy_scales = [&](uint32_t group) {
        const uint32_t to = lds_address(scales) + (group & 1) * T::SCALES;
        for (uint32_t q0 = 64 * wave; q0 < (uint32_t)T::WORDS; q0 += T::THREADS) {
            const uint32_t q = q0 + lane;
            const uint8_t *from = word_of(q < (uint32_t)T::WORDS ? q : 0, group);
            if (q < (uint32_t)T::WORDS && !(words && q % T::WPR == T::WPR - 1)) copy_word_to_lds(from, to + 4 * q0);
        }
    };
    const uint32_t row_shift_a = T::BYTES ? (uint32_t)((uintptr_t)p.SA & 3) : 0u, row_shift_w = (uint32_t)((uintptr_t)p.SW & 3);

    constexpr int MT = TM / 16, NT = TN / 16;
    const uint32_t block = wave % T::BLOCKS, kw = wave / T::BLOCKS, wm = (block % T::BLOCKS_M) * TM, wn = (block / T::BLOCKS_M) * TN;
    const uint32_t rot = (r >> 1) & 7;                                 // (tiles begin at multiples of 16 rows)
    f32x4 acc[NT][MT];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[j][i] = f32x4{0, 0, 0, 0};

    // byte of a row's first staged scale: its words, and where in them the row's bytes begin
    uint32_t at_w[NT], at_a[T::BYTES ? MT : 1];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const uint32_t row = wn + 16 * j + r, n = n0 + row < p.n ? n0 + row : p.n - 1;
        at_w[j] = ((T::BYTES ? BM : 0) + row) * (4 * T::WPR) + (T::IN_REGISTERS ? 0u : (row_shift_w + n * row_scales) & 3) + (T::BYTES ? g : SF == MMAEMU_SCALE_FORMAT_E8M0 ? g / 2 : g);
    }
    if constexpr (T::BYTES) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const uint32_t row = wm + 16 * i + r, m = m0 + row < p.m ? m0 + row : p.m - 1;
            at_a[i] = row * (4 * T::WPR) + (T::IN_REGISTERS ? 0u : (row_shift_a + m * row_scales) & 3) + g;
        }
    }

    // What a wavefront holds of its part of a step: weights as they are stored, their scales, and activations.
    struct Part {
        u32x4 wf[T::BYTES ? NT : 1], x[MT][2];
        u32x2 c[T::BYTES ? 1 : NT];
        uint32_t ws[NT], xs[T::BYTES ? MT : 1];
    };
    auto read_part = [&](Part &q, uint32_t s) {
        const uint8_t *a = lds + (s % S) * T::STAGE + kw * T::A_PART + (wm + r) * 128, *w = lds + (s % S) * T::STAGE + T::A_BYTES + kw * T::W_PART + (wn + r) * T::WB;
        const uint8_t *sc = scales + ((s / T::GROUP) & 1) * T::SCALES + (s % T::GROUP * WK + kw) * T::SB;
        w += T::BYTES ? 16 * (g ^ (r >> 2)) : 8 * g;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            if constexpr (T::BYTES) q.wf[j] = *reinterpret_cast<const u32x4 *>(w + 16 * T::WB * j);
            else q.c[j] = *reinterpret_cast<const u32x2 *>(w + 16 * T::WB * j);
            q.ws[j] = sc[at_w[j]];
        }
        const uint8_t *lo = a + 16 * ((T::BYTES ? g : 2 * g) ^ rot), *hi = a + 16 * ((T::BYTES ? 4 + g : 2 * g + 1) ^ rot);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            q.x[i][0] = *reinterpret_cast<const u32x4 *>(lo + 2048 * i);
            q.x[i][1] = *reinterpret_cast<const u32x4 *>(hi + 2048 * i);
            if constexpr (T::BYTES) q.xs[i] = sc[at_a[i]];
        }
    };
    auto multiply = [&](const Part &q) {
        if constexpr (T::BYTES) {
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                const i32x8 x = {(int)q.x[i][0][0], (int)q.x[i][0][1], (int)q.x[i][0][2], (int)q.x[i][0][3], (int)q.x[i][1][0], (int)q.x[i][1][1], (int)q.x[i][1][2], (int)q.x[i][1][3]};
#pragma unroll
                for (int j = 0; j < NT; ++j) acc[j][i] = mfma_scaled<AT>(q.wf[j], q.ws[j], x, q.xs[i], acc[j][i]);
            }
        } else {
            bool held = true;
            if constexpr (AT == MMAEMU_FP16 && SF == MMAEMU_SCALE_FORMAT_E8M0)
#pragma unroll
                for (int j = 0; j < NT; ++j) held = held && fp16_holds(q.ws[j]);
            if (__all(held)) {
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    f16x2 sh = {0, 0};
                    if constexpr (SF == MMAEMU_SCALE_FORMAT_UE4M3) sh = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(q.ws[j] & 0x7Fu, 1.0f, 0);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        Frag16 f;
                        if constexpr (SF == MMAEMU_SCALE_FORMAT_UE4M3) {
                            if constexpr (AT == MMAEMU_FP16) f = weights_fp16_by(q.c[j][h], f16x2{sh[0], sh[0]});
                            else f = weights_bf16_by(q.c[j][h], (float)sh[0]);
                        } else if constexpr (AT == MMAEMU_FP16) f = weights_fp16(q.c[j][h], q.ws[j]);
                        else f = weights_bf16(q.c[j][h], q.ws[j]);
#pragma unroll
                        for (int i = 0; i < MT; ++i) acc[j][i] = AT == MMAEMU_FP16 ? mfma_fp16(f, Frag16{q.x[i][h]}, acc[j][i]) : mfma_bf16(f, Frag16{q.x[i][h]}, acc[j][i]);
                    }
                }
            } else if constexpr (AT == MMAEMU_FP16 && SF == MMAEMU_SCALE_FORMAT_E8M0) {
#pragma unroll
                for (int j = 0; j < NT; ++j) {
                    const bool far = q.ws[j] - 253u < 2u;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const Frag16 f = weights_bf16(q.c[j][h], far ? q.ws[j] - 2 : q.ws[j]);
#pragma unroll
                        for (int i = 0; i < MT; ++i) {
                            // (rare: one piece at a time in registers, and nothing kept of it for the next weights)
                            Frag16 x = {q.x[i][h]}, hi, lo;
                            asm volatile("" : "+v"(x.w));
                            split_fp16(x, far ? 4.0f : 1.0f, hi, lo);
                            acc[j][i] = mfma_bf16(f, lo, acc[j][i]);
                            acc[j][i] = mfma_bf16(f, hi, acc[j][i]);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                }
            }
        }
    };

    static_assert(T::IN_REGISTERS || T::GROUP >= S - 2, "scales come in time");
    // Before step s is read: its copies have come, in all wavefronts; those of the S - 2 steps after it may be under way.  A group's
    // scales are copied in the group before, at least S - 2 steps ahead, so that this wait covers them.
    auto arrive = [&](uint32_t s) {
        if (s % T::GROUP == 0 && s && !copies_do(s / T::GROUP)) put_scales(s / T::GROUP);       // (into the half that was read a group ago)
        const uint32_t after = s + 1 < full ? full - 1 - s : 0;
        if (after >= S - 2) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((S - 2) * T::COPIES) : "memory");
        else if (S > 3 && after >= 2) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * T::COPIES) : "memory");
        else if (S > 3 && after == 1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(T::COPIES) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (s == full) {                                               // the step that ends inside: products beyond the row are zero times zero
#pragma unroll
            for (int i = 0; i < T::COPIES; ++i) {
                u32x4 v = {0, 0, 0, 0};
                if (s * T::KS + product_of(i) < p.k) v = *reinterpret_cast<const u32x4 *>(src[i] + (uint64_t)s * (i < T::AC ? 128 * WK : T::WB * WK));
                *reinterpret_cast<u32x4 *>(lds + (s % S) * T::STAGE + (i < T::AC ? 0 : T::A_BYTES) + 16 * chunk_of(i)) = v;
            }
            __syncthreads();
        }
        if (s % T::GROUP == 0 && s + T::GROUP < steps) {
            if constexpr (T::IN_REGISTERS) load_scales(s / T::GROUP + 1);
            else if (copies_do(s / T::GROUP + 1)) copy_scales(s / T::GROUP + 1);
        }
    };
    if constexpr (T::IN_REGISTERS) load_scales(0);
    put_scales(0);
    if constexpr (PIPE) {
        // The part of step s + 1 is read into registers before the products of step s, whose buffer then takes the copies of
        // step s + S.
#pragma unroll
        for (int s = 0; s < S; ++s)
            if (s < (int)full) issue(s);
        Part one, two;
        arrive(0);                                                     // (waits for one step more than it has to)
        read_part(one, 0);
        auto step = [&](uint32_t s, const Part &now, Part &next) {
            if (s + 1 < steps) {
                arrive(s + 1);
                read_part(next, s + 1);
                if (s + S < full) issue(s + S);
            }
            multiply(now);
        };
        for (uint32_t s = 0; s < steps; s += 2) {
            step(s, one, two);
            if (s + 1 < steps) step(s + 1, two, one);
        }
    } else {
#pragma unroll
        for (int s = 0; s < S - 1; ++s)
            if (s < (int)full) issue(s);
        for (uint32_t s = 0; s < steps; ++s) {
            arrive(s);
            if (s + S - 1 < full) issue(s + S - 1);                    // into the buffer that all have left
            Part q;
            read_part(q, s);
            multiply(q);
        }
    }
    if constexpr (WK > 1) {                                            // the sums of the wavefronts that share a block
        __syncthreads();
        f32x4 *sums = reinterpret_cast<f32x4 *>(lds) + block * (MT * NT * 64) + lane;
        if (kw)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int i = 0; i < MT; ++i) sums[((kw - 1) * T::BLOCKS * MT * NT + j * MT + i) * 64] = acc[j][i];
        __syncthreads();
        if (kw) return;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int q = 0; q < WK - 1; ++q) acc[j][i] += sums[(q * T::BLOCKS * MT * NT + j * MT + i) * 64];
    }
    with_output_type(p.d_type, [&](auto dt) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < MT; ++i) store_outputs<dt.value>(p, m0 + wm + 16 * i + r, n0 + wn + 16 * j + 4 * g, acc[j][i]);
    });
}

template <int AT, int SF, int BM, int BN, int TM, int TN, int WK, int S, bool PIPE> static mmaemu_status launch_tile(const ProductArgs &p, hipStream_t s)
{
    typedef Tile<AT, SF, BM, BN, TM, TN, WK, S> T;
    const uint32_t tm = (p.m + BM - 1) / BM, tn = (p.n + BN - 1) / BN;
    static_assert(T::LDS <= 160 * 1024 && (T::A_BYTES / 16) % 64 == 0 && (T::W_BYTES / 16) % 64 == 0, "tile");
    hipLaunchKernelGGL((tiled_kernel<AT, SF, BM, BN, TM, TN, WK, S, PIPE>), dim3(tm * tn), dim3(T::THREADS), T::LDS, s, p, tm, tn);
    MMAEMU_HIP(hipGetLastError());
    return MMAEMU_OK;
}

// Which block: the one whose rounds of workgroups over the 256 compute units take least, by what a round of each took (us for
// 8192 products, 8- and 16-bit activations, with all units at work).  A larger block reads less per product, a smaller one
// fills the chip with fewer rows; both sides were measured at the places where the choice changes, E4M3 and BF16 activations
// on MXFP4 weights, times in us:
//   m = 2048, n = 8192, k = 4096: 256 x 256 70 and 124, 128 x 256 79 and 148;   m = 256, n = 28672, k = 8192: 128 x 256 77 and 144, 256 x 256 121 and 223
//   m = 512, n = 8192, k = 8192: 128 x 128 45 and 72, 64 x 64 76 and 113;       m = 128, n = 8192, k = 8192: 64 x 64 21 and 31, 32 x 64 25 and 31
//   m = 64, n = 8192, k = 8192: 32 x 64 15 and 22, 64 x 64 20 and 29;           m = 32, n = 8192, k = 8192: 32 x 32 11 and 14, 32 x 64 14 and 22
struct BlockChoice { uint32_t bm, bn; float one[2], two[2]; };         // two: of 512 workgroups (two of the 32 x 64 ones fit a unit)
static const BlockChoice BLOCK_CHOICES[] = {
    {256, 256, {119, 223}, {238, 446}}, {128, 256, {72, 139}, {144, 278}}, {128, 128, {45, 72}, {90, 144}},
    {64, 64, {21, 30}, {42, 60}},       {32, 64, {14.5f, 22}, {26, 31}},   {32, 32, {11, 14}, {22, 28}},
};

static uint32_t choose_block(uint32_t m, uint32_t n, bool bytes, bool fp16_e8m0)
{
    uint32_t best = 0;
    float least = 0;
    for (uint32_t i = fp16_e8m0 ? 1 : 0; i < sizeof(BLOCK_CHOICES) / sizeof(BLOCK_CHOICES[0]); ++i) {      // (FP16 activations' second way leaves too few registers for 256 x 256)
        const BlockChoice &b = BLOCK_CHOICES[i];
        const uint64_t tiles = (uint64_t)((m + b.bm - 1) / b.bm) * ((n + b.bn - 1) / b.bn);
        const uint64_t rounds = (tiles + 255) / 256;
        const float t = b.two[bytes ? 0 : 1] * (float)(rounds / 2) + (rounds % 2 ? b.one[bytes ? 0 : 1] : 0.0f);
        if (least == 0 || t < least) {
            least = t;
            best = i;
        }
    }
    return best;
}

const char *tiled_name(uint32_t m, uint32_t n, uint32_t a_type, uint32_t scale_format)
{
    static const char *const names[] = {"blocks of 256 x 256", "blocks of 128 x 256", "blocks of 128 x 128", "blocks of 64 x 64", "blocks of 32 x 64", "blocks of 32 x 32"};
    return names[choose_block(m, n, is_byte_type(a_type), a_type == MMAEMU_FP16 && scale_format == MMAEMU_SCALE_FORMAT_E8M0)];
}

template <int AT, int SF> static mmaemu_status launch_tiled_typed(const ProductArgs &p, hipStream_t s)
{
    constexpr bool BYTES = AT == MMAEMU_FP8_E4M3 || AT == MMAEMU_FP8_E5M2, TWO_WAYS = AT == MMAEMU_FP16 && SF == MMAEMU_SCALE_FORMAT_E8M0;
    switch (choose_block(p.m, p.n, BYTES, TWO_WAYS)) {
    case 0:
        // (BF16 weights under UE4M3 scales take four instructions a pair: blocks of fewer weights per wavefront, 200 -> 157 us at
        // 2048 x 8192 x 4096)
        if constexpr (AT == MMAEMU_BF16 && SF == MMAEMU_SCALE_FORMAT_UE4M3) return launch_tile<AT, SF, 256, 256, 128, 64, 1, 3, false>(p, s);
        else if constexpr (!TWO_WAYS) return launch_tile<AT, SF, 256, 256, 64, 128, 1, 3, false>(p, s);
    case 1: return launch_tile<AT, SF, 128, 256, 64, 64, 1, 3, !TWO_WAYS>(p, s);
    case 2: return launch_tile<AT, SF, 128, 128, 64, 64, 2, 2, !TWO_WAYS>(p, s);
    case 3:
        if constexpr (BYTES) return launch_tile<AT, SF, 64, 64, 32, 32, 4, 2, false>(p, s);
        else return launch_tile<AT, SF, 64, 64, 64, 32, 4, 2, false>(p, s);
    case 4: return launch_tile<AT, SF, 32, 64, 32, 32, 4, 3, false>(p, s);
    default: return launch_tile<AT, SF, 32, 32, 32, 32, 8, 3, false>(p, s);
    }
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
