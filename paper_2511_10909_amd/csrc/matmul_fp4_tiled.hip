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
    static constexpr bool IN_REGISTERS = SB * WK <= 4;                 // scales staged through registers (else by copies, as aligned words)
    static constexpr int GB = SB * WK < 16 ? 16 : SB * WK, GROUP = GB / (SB * WK);     // scale bytes of a row staged together, and their steps
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

// waits until at most `steps` (up to MOST) steps of EACH copies, of those issued last, are under way
template <int MOST, int EACH> __device__ __forceinline__ void wait_copies(uint32_t steps)
{
    if constexpr (MOST > 0) {
        if (steps < MOST) return wait_copies<MOST - 1, EACH>(steps);
    }
    static_assert(MOST * EACH < 64, "the counter's range");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(MOST * EACH) : "memory");
}

// How a wavefront's reads from LDS and its matrix instructions follow one another: a step's reads before its products; the next step's reads
// before them; or the workgroup's eight wavefronts in two halves, one of each on every SIMD, that take turns: while one reads, the other
// multiplies (8192 x 8192 outputs, 8192 products, in order and by turns: E4M3 437 -> 403 us, BF16 872 -> 789 in 256 x 256; 252 -> 244
// and, from reading ahead, 480 -> 475 for half the rows in 128 x 256).
enum class Order { PLAIN, AHEAD, TURNS };

template <int AT, int SF, int BM, int BN, int TM, int TN, int WK, int S, Order ORDER>
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
    const uint32_t steps = (p.k + T::KS - 1) / T::KS, row_scales = p.k / T::PER_SCALE;
    const bool ends_inside = steps * T::KS > p.k;                      // the last step: products beyond the row are zero times zero

    // Source of each of this thread's copies, from the block's first row: part, row, 16-byte chunk of it.  Chunks are stored where
    // lds_rotation puts them.
    uint32_t src[T::COPIES];
    auto chunk_of = [&](int i) MMAEMU_INLINE -> uint32_t { return i < T::AC ? (i * T::THREADS + tid) % (T::A_BYTES / 16) : ((i - T::AC) * T::THREADS + tid) % (T::W_BYTES / 16); };
    auto product_of = [&](int i) MMAEMU_INLINE -> uint32_t {                         // the chunk's first product within the step
        const uint32_t q = chunk_of(i);
        if (i < T::AC) return T::PART * (q / (T::A_PART / 16)) + (T::BYTES ? 16 : 8) * ((q % 8) ^ lds_rotation<8>(q / 8));
        return T::PART * (q / (T::W_PART / 16)) + 32 * (T::BYTES ? (q % 4) ^ lds_rotation<4>(q / 4) : (q % 2) ^ lds_rotation<2>(q / 2));
    };
    const uint32_t rows_m = p.m - m0 < BM ? p.m - m0 : BM, rows_n = p.n - n0 < BN ? p.n - n0 : BN;      // (rows beyond: the last one again)
#pragma unroll
    for (int i = 0; i < T::COPIES; ++i) {
        if (i < T::AC) {
            const uint32_t row = chunk_of(i) % (T::A_PART / 16) / 8;
            src[i] = (row < rows_m ? row : rows_m - 1) * (uint32_t)p.a_stride + product_of(i) * (T::BYTES ? 1 : 2);
        } else {
            const uint32_t row = chunk_of(i) % (T::W_PART / 16) / (T::WB / 16);
            src[i] = (row < rows_n ? row : rows_n - 1) * (p.k / 2) + product_of(i) / 2;
        }
    }
    // The next step that copies are issued for: its place in both operands and in LDS.
    const uint8_t *next_a = p.A + (uint64_t)m0 * p.a_stride, *next_w = p.W + (uint64_t)n0 * (p.k / 2);
    uint32_t next_step = 0, next_at = 0;
    auto issue = [&](bool whole) MMAEMU_INLINE {
        auto place = [&](int i) MMAEMU_INLINE -> uint32_t {                          // of this wavefront's first chunk
            return 16 * (i < T::AC ? (i * T::THREADS + 64 * wave) % (T::A_BYTES / 16) : T::A_BYTES / 16 + ((i - T::AC) * T::THREADS + 64 * wave) % (T::W_BYTES / 16));
        };
        if (whole) {
#pragma unroll
            for (int i = 0; i < T::COPIES; ++i) copy_to_lds(i < T::AC ? next_a : next_w, src[i], lds_address(lds) + next_at + place(i));
        } else {
#pragma unroll
            for (int i = 0; i < T::COPIES; ++i) {
                if (next_step * T::KS + product_of(i) < p.k) copy_to_lds(i < T::AC ? next_a : next_w, src[i], lds_address(lds) + next_at + place(i));
                else *reinterpret_cast<u32x4 *>(lds + next_at + place(i) + 16 * lane) = u32x4{0, 0, 0, 0};
            }
        }
        next_a += 128 * WK;
        next_w += T::WB * WK;
        next_step += 1;
        next_at = next_at == (S - 1) * T::STAGE ? 0 : next_at + T::STAGE;
    };
    const uint32_t whole_steps = ends_inside ? steps - 1 : steps;

    // Scales, GB bytes of a row at a time.  Where that is four steps and more, a thread loads a row's into registers in the group
    // before and stores them at the barrier before the group; the compiler then waits for the copies under way as well, which costs less
    // than the instructions of the other way (8192^3, E4M3: 430 against 470 us).  Where it is fewer, copies bring the aligned
    // words that hold them (a row begins at any byte; reads are of bytes).  Bytes beyond a row are 2^0 (they meet zeros).
    constexpr uint32_t ONES = SF == MMAEMU_SCALE_FORMAT_UE4M3 ? 0x38383838u : 0x7F7F7F7Fu;
    constexpr int REGS = T::IN_REGISTERS ? (T::SCALE_ROWS + T::THREADS - 1) / T::THREADS : (T::WORDS + T::THREADS - 1) / T::THREADS;
    // rows or words of this thread: their rows' beginnings, and where their next group begins (words: at the aligned word that
    // holds its first byte)
    const uint8_t *sbegin[REGS], *sfrom[REGS];
#pragma unroll
    for (int i = 0; i < REGS; ++i) {
        const uint32_t q = i * T::THREADS + tid, all = T::IN_REGISTERS ? T::SCALE_ROWS : T::WORDS, c = q < all ? q : 0;
        const uint32_t srow = T::IN_REGISTERS ? c : c / T::WPR, row_n = srow - (T::BYTES ? BM : 0);      // of activations, then of weights
        sbegin[i] = p.SW + (uint64_t)(n0 + (row_n < rows_n ? row_n : rows_n - 1)) * row_scales;
        if constexpr (T::BYTES) {
            const uint8_t *of_a = p.SA + (uint64_t)(m0 + (srow < rows_m ? srow : rows_m - 1)) * row_scales;
            sbegin[i] = srow < (uint32_t)BM ? of_a : sbegin[i];
        }
        sfrom[i] = sbegin[i];
        if (!T::IN_REGISTERS) sfrom[i] += 4 * (c % T::WPR) - ((uintptr_t)sfrom[i] & 3);
    }
    uint32_t next_group = 0;                       // the group that sfrom points at
    Words4<1> sreg[T::IN_REGISTERS ? REGS : 1];
    uint32_t wreg[T::IN_REGISTERS ? 1 : REGS];
    auto load_scales = [&]() MMAEMU_INLINE {                     // the next group into registers, byte by byte where a word is not all of its row
#pragma unroll
        for (int i = 0; i < REGS; ++i) {
            if constexpr (T::IN_REGISTERS) {
                if (16 * next_group + 16 <= row_scales) sreg[i] = *reinterpret_cast<const Words4<1> *>(sfrom[i]);
                else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) sreg[i].w[e] = ONES;
#pragma unroll
                    for (uint32_t e = 0; e < 15; ++e)
                        if (16 * next_group + e < row_scales) sreg[i].w[e / 4] = (sreg[i].w[e / 4] & ~(0xFFu << (8 * (e % 4)))) | (uint32_t)sfrom[i][e] << (8 * (e % 4));
                }
            } else {
                const uint8_t *begin = sbegin[i], *end = begin + row_scales, *from = sfrom[i];
                wreg[i] = ONES;
                if (from >= begin && from + 4 <= end) wreg[i] = *reinterpret_cast<const uint32_t *>(from);
                else
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (from + e >= begin && from + e < end) wreg[i] = (wreg[i] & ~(0xFFu << (8 * e))) | (uint32_t)from[e] << (8 * e);
            }
        }
#pragma unroll
        for (int i = 0; i < REGS; ++i) sfrom[i] += T::GB;
        next_group += 1;
    };
    auto put_scales = [&](uint32_t half) MMAEMU_INLINE {         // what load_scales has loaded
#pragma unroll
        for (int i = 0; i < REGS; ++i) {
            const uint32_t q = i * T::THREADS + tid;
            if constexpr (T::IN_REGISTERS) {
                if (T::SCALE_ROWS % T::THREADS == 0 || q < (uint32_t)T::SCALE_ROWS) {
                    // (rows eight apart would meet in a bank: every other eight has its words exchanged in pairs)
                    const bool swap = (q & 8) != 0;
                    const uint32_t *w = sreg[i].w;
                    *reinterpret_cast<u32x4 *>(scales + half + 16 * q) = u32x4{swap ? w[1] : w[0], swap ? w[0] : w[1], swap ? w[3] : w[2], swap ? w[2] : w[3]};
                }
            } else if (T::WORDS % T::THREADS == 0 || q < (uint32_t)T::WORDS) *reinterpret_cast<uint32_t *>(scales + half + 4 * q) = wreg[i];
        }
    };
    // copies do it where all words lie within their rows (with rows of aligned words the last is not needed)
    const bool words = row_scales % 4 == 0 && ((uintptr_t)p.SW & 3) == 0 && (!T::BYTES || ((uintptr_t)p.SA & 3) == 0);
    const uint32_t reach = words ? T::GB : T::GB + 4, copied_groups = T::IN_REGISTERS || row_scales < reach ? 0 : (row_scales - reach) / T::GB + 1;
    auto copy_scales = [&](uint32_t half) MMAEMU_INLINE {
#pragma unroll
        for (int i = 0; i < REGS; ++i) {
            const uint32_t q = i * T::THREADS + tid;
            if ((T::WORDS % T::THREADS == 0 || q < (uint32_t)T::WORDS) && !(words && q % T::WPR == T::WPR - 1)) copy_word_to_lds(sfrom[i], lds_address(scales) + half + 4 * (i * T::THREADS + 64 * wave));
            sfrom[i] += T::GB;
        }
        next_group += 1;
    };

    constexpr int MT = TM / 16, NT = TN / 16;
    const uint32_t block = wave % T::BLOCKS, kw = wave / T::BLOCKS, wm = (block % T::BLOCKS_M) * TM, wn = (block / T::BLOCKS_M) * TN;
    const uint32_t rot = lds_rotation<8>(r);                                // (tiles begin at multiples of 16 rows)
    f32x4 acc[NT][MT];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[j][i] = f32x4{0, 0, 0, 0};

    // byte of a row's first staged scale: its words, and where in them the row's bytes begin (the same for rows 16 apart)
    const uint32_t row_w = wn + r, row_a = wm + r;
    const uint32_t at_w = ((T::BYTES ? BM : 0) + row_w) * (4 * T::WPR) + (T::IN_REGISTERS ? 0u : ((uint32_t)(uintptr_t)p.SW + (n0 + row_w) * row_scales) & 3) +
                          kw * T::SB + (T::BYTES ? g : SF == MMAEMU_SCALE_FORMAT_E8M0 ? g / 2 : g);
    const uint32_t at_a = T::BYTES ? row_a * (4 * T::WPR) + (T::IN_REGISTERS ? 0u : ((uint32_t)(uintptr_t)p.SA + (m0 + row_a) * row_scales) & 3) + kw * T::SB + g : 0u;

    // What a wavefront holds of its part of a step: weights as they are stored, their scales, and activations.
    struct Part {
        u32x4 wf[T::BYTES ? NT : 1], x[MT][2];
        u32x2 c[T::BYTES ? 1 : NT];
        uint32_t ws[NT], xs[T::BYTES ? MT : 1];
    };
    const uint32_t in_a = kw * T::A_PART + (wm + r) * 128, in_w = T::A_BYTES + kw * T::W_PART + (wn + r) * T::WB + (T::BYTES ? 16 * (g ^ lds_rotation<4>(r)) : 16 * ((g >> 1) ^ lds_rotation<2>(r)) + 8 * (g & 1));
    const uint32_t in_lo = in_a + 16 * ((T::BYTES ? g : 2 * g) ^ rot), in_hi = in_a + 16 * ((T::BYTES ? 4 + g : 2 * g + 1) ^ rot);
    const uint32_t swapped = T::IN_REGISTERS ? (r & 8) / 2 : 0u;
    auto read_part = [&](Part &q, uint32_t at, uint32_t half, uint32_t in_group) MMAEMU_INLINE {       // of the step in the buffer `at`, its scales in that half
        const uint32_t sc = half + ((in_group * (WK * T::SB)) ^ swapped);
        const uint8_t *w = lds + at + in_w, *lo = lds + at + in_lo, *hi = lds + at + in_hi, *sw = scales + sc + at_w, *sa = scales + sc + at_a;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            if constexpr (T::BYTES) q.wf[j] = *reinterpret_cast<const u32x4 *>(w + 16 * T::WB * j);
            else q.c[j] = *reinterpret_cast<const u32x2 *>(w + 16 * T::WB * j);
            q.ws[j] = sw[64 * T::WPR * j];
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            q.x[i][0] = *reinterpret_cast<const u32x4 *>(lo + 2048 * i);
            q.x[i][1] = *reinterpret_cast<const u32x4 *>(hi + 2048 * i);
            if constexpr (T::BYTES) q.xs[i] = sa[64 * T::WPR * i];
        }
    };
    auto multiply = [&](const Part &q) MMAEMU_INLINE {
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
                    const bool far = any_far(q.ws[j]);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const Frag16 f = weights_second_way(q.c[j][h], q.ws[j], far);
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

    static_assert(T::IN_REGISTERS || T::GROUP >= S - 2, "a group's scales have come with the step that they are first read in");
    // The step that is read next: its buffer and its place among the scales.
    uint32_t at = 0, in_group = 0, half = 0;
    auto go_on = [&]() MMAEMU_INLINE {
        at = at == (S - 1) * T::STAGE ? 0 : at + T::STAGE;
        if (++in_group == T::GROUP) {
            in_group = 0;
            half ^= T::SCALES;
        }
    };
    // Before step s is read: its copies have come, in all wavefronts; those of the S - 2 steps after it may be under way.  A group's
    // scales are copied in the group before, at least S - 2 steps ahead, so that this wait covers them.  (STEADY: away from the
    // end, where nothing has to be asked.)
    auto arrive = [&](uint32_t s, auto steady) MMAEMU_INLINE {
        if constexpr (steady && !T::IN_REGISTERS) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((S - 2) * T::COPIES) : "memory");
        else {
            if (in_group == 0 && s && s / T::GROUP >= copied_groups) put_scales(half);         // (into the half that was read a group ago)
            // (a step that ends inside counts as none: it may have fewer copies)
            wait_copies<S - 2, T::COPIES>(steady || s + (S - 2) < whole_steps ? S - 2 : s < whole_steps ? whole_steps - 1 - s : 0);
        }
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (in_group == 0 && (steady || s + T::GROUP < steps)) {
            if (!T::IN_REGISTERS && (steady || s / T::GROUP + 1 < copied_groups)) copy_scales(half ^ T::SCALES);
            else load_scales();
        }
    };
    // steps before which all that is waited for or issued is whole
    constexpr bool PIPE = ORDER == Order::AHEAD;
    constexpr uint32_t AHEAD = PIPE ? S : S - 1;   // steps issued ahead of the one that is multiplied
    uint32_t steady_steps = whole_steps > AHEAD ? whole_steps - AHEAD : 0;
    if (!T::IN_REGISTERS) {
        const uint32_t last = copied_groups > 1 ? (copied_groups - 1) * T::GROUP : 0;
        if (last < steady_steps + (PIPE ? 1 : 0)) steady_steps = PIPE ? (last ? last - 1 : 0) : last;
    } else if (steady_steps * T::SB * WK + 32 > row_scales) steady_steps = row_scales >= 32 ? (row_scales - 32) / (T::SB * WK) : 0;
    load_scales();
#pragma unroll
    for (uint32_t s = 0; s < AHEAD; ++s)
        if (s < steps) issue(s < whole_steps);
    put_scales(0);
    uint32_t s = 0;
    if constexpr (PIPE) {
        // The part of step s + 1 is read into registers before the products of step s, whose buffer then takes the copies of
        // step s + S.
        Part one, two;
        arrive(0, std::false_type());                                  // (waits for one step more than it has to)
        read_part(one, at, half, in_group);
        auto step = [&](const Part &now, Part &next, auto steady) MMAEMU_INLINE {
            if (steady || s + 1 < steps) {
                go_on();
                arrive(s + 1, steady);
                read_part(next, at, half, in_group);
                if (steady || s + S < steps) issue(steady || s + S < whole_steps);
            }
            multiply(now);
            ++s;
        };
        while (s + 1 < steady_steps) {
            step(one, two, std::true_type());
            step(two, one, std::true_type());
        }
        while (s < steps) {
            step(one, two, std::false_type());
            if (s < steps) step(two, one, std::false_type());
        }
    } else if constexpr (ORDER == Order::TURNS) {
        static_assert(T::THREADS == 512 && S == 3 && T::IN_REGISTERS && T::GROUP > 1, "two halves of four wavefronts");
        // Between barriers 2 s and 2 s + 1 the first half reads step s and issues the copies of step s + 2, while the second multiplies
        // step s - 1; then they change places.  The copies go into the buffer of step s - 1, which the second half has read before barrier
        // 2 s.  What step s + 1 needs of a wavefront (its copies, its scales) is there before barrier 2 s + 2.
        const bool second = wave >= 4;
        auto turn = [&]() MMAEMU_INLINE {
            __builtin_amdgcn_sched_barrier(0);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        };
        auto ready = [&](auto steady) MMAEMU_INLINE {            // what this wavefront brings for step s + 1
            wait_copies<1, T::COPIES>(steady || s + 2 < whole_steps ? 1 : 0);
            if (in_group == 0 && (steady || s + 1 + T::GROUP < steps)) load_scales();
        };
        auto step = [&](auto steady) MMAEMU_INLINE {
            if (in_group + 1 == T::GROUP && (steady || s + 1 < steps)) put_scales(half ^ T::SCALES);
            if (steady || s + 2 < steps) issue(steady || s + 2 < whole_steps);
            Part q;
            read_part(q, at, half, in_group);
            go_on();
            if (second) ready(steady);
            turn();
            multiply(q);
            if (!second) ready(steady);
            turn();
            ++s;
        };
        wait_copies<1, T::COPIES>(whole_steps > 1 ? 1 : 0);
        if (T::GROUP < steps) load_scales();
        turn();
        if (second) turn();
        while (s < steady_steps) step(std::true_type());
        while (s < steps) step(std::false_type());
        if (!second) turn();
    } else {
        auto step = [&](auto steady) MMAEMU_INLINE {
            arrive(s, steady);
            if (steady || s + S - 1 < steps) issue(steady || s + S - 1 < whole_steps);          // into the buffer that all have left
            Part q;
            read_part(q, at, half, in_group);
            go_on();
            multiply(q);
            ++s;
        };
        while (s < steady_steps) step(std::true_type());
        while (s < steps) step(std::false_type());
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

template <int AT, int SF, int BM, int BN, int TM, int TN, int WK, int S, Order ORDER> static mmaemu_status launch_tile(const ProductArgs &p, hipStream_t s)
{
    typedef Tile<AT, SF, BM, BN, TM, TN, WK, S> T;
    const uint32_t tm = (p.m + BM - 1) / BM, tn = (p.n + BN - 1) / BN;
    static_assert(T::LDS <= 160 * 1024 && (T::A_BYTES / 16) % 64 == 0 && (T::W_BYTES / 16) % 64 == 0, "tile");
    hipLaunchKernelGGL((tiled_kernel<AT, SF, BM, BN, TM, TN, WK, S, ORDER>), dim3(tm * tn), dim3(T::THREADS), T::LDS, s, p, tm, tn);
    MMAEMU_HIP(hipGetLastError());
    return MMAEMU_OK;
}

// Which block: the one whose rounds of workgroups over the 256 compute units take least, by what one round and two rounds took (us
// for 2048 and 8192 products, E4M3 and BF16 activations on MXFP4 weights, 8192 weight rows; of some blocks two workgroups fit a unit).
// Between and beyond these lengths the time is a straight line, below them that of 2048.  A larger block reads less per product, a smaller
// one fills the chip with fewer tokens and splits its products among more wavefronts.  Both sides where the choice changes, E4M3 and BF16, us:
//   2048 tokens, 8192 x 4096: 256 x 256 54 and 102, 128 x 256 66 and 122;  256 tokens, 28672 x 8192: 128 x 256 66 and 123, 256 x 256 100 and 198
//   512 tokens, 8192 x 8192: 128 x 128 36 and 63, 64 x 128 45 and 66;      8192 x 2048: 128 x 128 15 and 23, 64 x 128 17 and 21
//   256 tokens, 8192 x 8192: 64 x 128 23 and 36, 64 x 64 26 and 43, 128 x 128 35 and 61
//   128 tokens: 64 x 64 16 and 22, 32 x 64 21 and 26;  64 tokens: 32 x 64 12 and 16, 64 x 64 16 and 21, 32 x 32 15 and 22;  32 tokens: 32 x 32 9.5 and 12, 32 x 64 12 and 16
// The other kinds go by the same times: on nineteen sizes of 64 to 4096 tokens FP16 on NVFP4 took at most 6 % more than in its fastest block, BF16 on
// NVFP4 6 (256 tokens, 28672 x 8192: 190 us, 180 in the same blocks unsplit), FP16 on MXFP4 11 (1024 tokens, 4096 x 4096: 64 x 128 49, 128 x 128 44).
struct BlockTimes { float one[2], two[2]; };       // [0]: 8-bit activations, [1]: 16-bit ones
struct BlockChoice { uint32_t bm, bn; BlockTimes at_2048, at_8192; };
static const BlockChoice BLOCK_CHOICES[] = {
    {256, 256, {{33.5f, 58}, {64, 111}}, {{94, 190}, {193, 376}}},
    {128, 256, {{22.5f, 35.5f}, {40.4f, 67}}, {{60, 113}, {116, 232}}},
    {128, 128, {{14.9f, 23}, {25.9f, 42.6f}}, {{35.5f, 63}, {69, 123}}},
    {64, 128, {{9.8f, 13.2f}, {17.2f, 20.9f}}, {{22.9f, 35.5f}, {44.5f, 66}}},
    {64, 64, {{7.3f, 11.2f}, {9.9f, 17.9f}}, {{15.8f, 22.3f}, {26.2f, 42.5f}}},
    {32, 64, {{5.8f, 7.5f}, {9.8f, 9.7f}}, {{11.8f, 15.9f}, {21.4f, 25.8f}}},
    {32, 32, {{5.1f, 6.8f}, {8, 10.6f}}, {{9.5f, 11.8f}, {15, 21.6f}}},
};
constexpr uint32_t BLOCK_KINDS = sizeof(BLOCK_CHOICES) / sizeof(BLOCK_CHOICES[0]), UNITS = 256;

static uint32_t blocks_along(uint32_t size, uint32_t block) { return (size + block - 1) / block; }

static float block_time(const BlockChoice &b, uint32_t m, uint32_t n, uint32_t k, bool bytes)
{
    const uint64_t rounds = ((uint64_t)blocks_along(m, b.bm) * blocks_along(n, b.bn) + UNITS - 1) / UNITS;
    const int type = bytes ? 0 : 1;
    const auto of = [&](const BlockTimes &t) { return t.two[type] * (float)(rounds / 2) + (rounds % 2 ? t.one[type] : 0.0f); };
    const float brief = of(b.at_2048), slope = (of(b.at_8192) - brief) / 6144;
    return k > 2048 ? brief + slope * (float)(k - 2048) : brief;
}

// `time`: what it takes; FP16 activations' second way under E8M0 scales leaves too few registers for 256 x 256
static uint32_t choose_block(uint32_t m, uint32_t n, uint32_t k, bool bytes, bool fp16_e8m0, float *time = nullptr)
{
    uint32_t best = fp16_e8m0 ? 1 : 0;
    float least = block_time(BLOCK_CHOICES[best], m, n, k, bytes);
    for (uint32_t i = best + 1; i < BLOCK_KINDS; ++i) {
        const float t = block_time(BLOCK_CHOICES[i], m, n, k, bytes);
        if (t < least) {
            least = t;
            best = i;
        }
    }
    if (time) *time = least;
    return best;
}

// Blocks that fill some rounds and leave a few for one more cost that whole round.  Where it takes less, whole rounds go first, as a
// product with fewer weight rows or tokens, and what is left follows in blocks of its own choice, in a second launch; the parts have to be
// expected to take a twentieth less, and 3 us (1294 E5M2 tokens, 24384 x 5568: 252 us in one launch, 188 in two; 6639 E4M3 tokens, 2432 x 1888:
// 59 and 45; but 1648 BF16 tokens, 3010 x 544: 15.6 and 18.4).
struct Split { uint32_t m, n, block; };            // the first part (all of it: one launch)

static Split choose_split(uint32_t m, uint32_t n, uint32_t k, bool bytes, bool fp16_e8m0)
{
    float whole;
    Split best = {m, n, choose_block(m, n, k, bytes, fp16_e8m0, &whole)};
    const float few = 3.0f * (k < 2048 ? 2048.0f / (float)k : 1.0f);  // (block_time is that of 2048 products there)
    float least = whole - (few > 0.05f * whole ? few : 0.05f * whole);
    for (uint32_t i = fp16_e8m0 ? 1 : 0; i < BLOCK_KINDS; ++i) {
        const BlockChoice &b = BLOCK_CHOICES[i];
        const uint32_t tm = blocks_along(m, b.bm), tn = blocks_along(n, b.bn);
        const uint64_t rounds = (uint64_t)tm * tn / UNITS;
        const auto consider = [&](uint64_t m1, uint64_t n1) {
            if (!rounds || !m1 || !n1 || m1 > m || n1 > n || (m1 == m && n1 == n)) return;
            float rest;
            choose_block(m1 < m ? m - (uint32_t)m1 : m, n1 < n ? n - (uint32_t)n1 : n, k, bytes, fp16_e8m0, &rest);
            const float t = block_time(b, (uint32_t)m1, (uint32_t)n1, k, bytes) + rest;
            if (t < least) {
                least = t;
                best = {(uint32_t)m1, (uint32_t)n1, i};
            }
        };
        consider(m, UNITS * rounds / tm * b.bn);
        consider(UNITS * rounds / tn * b.bm, n);
    }
    return best;
}

static bool two_ways(uint32_t a_type, uint32_t scale_format) { return a_type == MMAEMU_FP16 && scale_format == MMAEMU_SCALE_FORMAT_E8M0; }

const char *tiled_name(uint32_t m, uint32_t n, uint32_t k, uint32_t a_type, uint32_t scale_format)
{
    static const char *const names[] = {"blocks of 256 x 256", "blocks of 128 x 256", "blocks of 128 x 128", "blocks of 64 x 128", "blocks of 64 x 64", "blocks of 32 x 64", "blocks of 32 x 32"};
    return names[choose_split(m, n, k, is_byte_type(a_type), two_ways(a_type, scale_format)).block];
}

template <int AT, int SF> static mmaemu_status launch_block(const ProductArgs &p, uint32_t block, hipStream_t s)
{
    constexpr bool BYTES = AT == MMAEMU_FP8_E4M3 || AT == MMAEMU_FP8_E5M2, TWO_WAYS = AT == MMAEMU_FP16 && SF == MMAEMU_SCALE_FORMAT_E8M0;
    switch (block) {
    // (the wavefront's share, the depth of the buffers and the reading ahead: what was fastest for each kind of activations; deeper buffers
    // than three gain nothing; wavefronts that take weights to 16 bits have fewer of them and more tokens: 2048 x 8192 x 4096 in
    // 64 x 128 and 128 x 64 a wavefront, under UE4M3 scales BF16 172 and 137 us, FP16 124 and 113, BF16 under E8M0 110 and 106; 8-bit ones have
    // no such work (55 and 58), and sixteen wavefronts in the smallest blocks: 64 E4M3 tokens on 8192 x 8192 12.7 ->
    // 11.8, 16-bit ones 16.2 -> 18.3; 128 BF16 tokens on 8192 x 8192 in 64 x 64: 30 us with 32 x 32 a wavefront, 22 with 64 x 32)
    case 0:
        if constexpr (BYTES) return launch_tile<AT, SF, 256, 256, 64, 128, 1, 3, Order::TURNS>(p, s);
        else if constexpr (!TWO_WAYS) return launch_tile<AT, SF, 256, 256, 128, 64, 1, 3, Order::TURNS>(p, s);
    case 1: return launch_tile<AT, SF, 128, 256, 64, 64, 1, 3, TWO_WAYS ? Order::PLAIN : Order::TURNS>(p, s);
    case 2: return launch_tile<AT, SF, 128, 128, 64, 64, 2, 3, !BYTES && !TWO_WAYS ? Order::AHEAD : Order::PLAIN>(p, s);
    case 3:
        // (one round: sixteen wavefronts a unit, 256 BF16 tokens on 8192 x 8192 39 -> 35 us; two: two workgroups of eight, 512 tokens 71 -> 66)
        if constexpr (!BYTES && !TWO_WAYS)
            if ((uint64_t)blocks_along(p.m, 64) * blocks_along(p.n, 128) <= UNITS) return launch_tile<AT, SF, 64, 128, 64, 32, 4, 3, Order::PLAIN>(p, s);
        return launch_tile<AT, SF, 64, 128, 64, 32, 2, TWO_WAYS ? 2 : 3, Order::PLAIN>(p, s);
    case 4:
        if constexpr (BYTES) return launch_tile<AT, SF, 64, 64, 32, 32, 2, 3, Order::PLAIN>(p, s);
        else return launch_tile<AT, SF, 64, 64, 64, 32, 4, 3, !TWO_WAYS ? Order::AHEAD : Order::PLAIN>(p, s);
    case 5: return launch_tile<AT, SF, 32, 64, 32, BYTES ? 16 : 32, 4, 3, Order::PLAIN>(p, s);
    default: return launch_tile<AT, SF, 32, 32, 32, BYTES ? 16 : 32, 8, 3, Order::PLAIN>(p, s);
    }
}

template <int AT, int SF> static mmaemu_status launch_tiled_typed(const ProductArgs &p, hipStream_t s)
{
    constexpr bool BYTES = AT == MMAEMU_FP8_E4M3 || AT == MMAEMU_FP8_E5M2, TWO_WAYS = AT == MMAEMU_FP16 && SF == MMAEMU_SCALE_FORMAT_E8M0;
    const Split first = choose_split(p.m, p.n, p.k, BYTES, TWO_WAYS);
    ProductArgs part = p;
    part.m = first.m;
    part.n = first.n;
    const mmaemu_status st = launch_block<AT, SF>(part, first.block, s);
    if (st != MMAEMU_OK || (first.m == p.m && first.n == p.n)) return st;
    const uint64_t eb = p.d_type == MMAEMU_FP32 ? 4 : 2;
    part = p;
    if (first.m < p.m) {
        part.m = p.m - first.m;
        part.A = p.A + first.m * p.a_stride;
        if (BYTES) part.SA = p.SA + (uint64_t)first.m * (p.k / 32);
        part.D = (char *)p.D + first.m * p.d_stride * eb;
    } else {
        part.n = p.n - first.n;
        part.W = p.W + (uint64_t)first.n * (p.k / 2);
        part.SW = p.SW + (uint64_t)first.n * (p.k / (SF == MMAEMU_SCALE_FORMAT_E8M0 ? 32 : 16));
        part.D = (char *)p.D + first.n * eb;
    }
    return launch_block<AT, SF>(part, choose_block(part.m, part.n, p.k, BYTES, TWO_WAYS), s);
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
