// Copies of pages within caches: a fork's last pages, a compaction's moves.
//
// Bound by memory: each byte is read and written once (150 pages of 69632 bytes in 16 layers: 68 us, 4.9 TB/s).  A workgroup copies a stretch of one page of one layer, 16 bytes a lane and four at once in flight;
// the moves travel as the kernel's argument, so a captured graph holds them.
#include "block_scale.hpp"

namespace mmaemu {

constexpr uint32_t COPY_MOVES = 440;               // of a launch: 8 bytes each within the 4 KB that a launch's arguments may take
constexpr uint32_t COPY_FEW = 32;                  // most calls' moves: the launch's arguments are 288 bytes then, not 3.5 KB (16 pages 5.7 us of the host, 5.9 with the larger ones)
constexpr uint32_t COPY_STRETCH = 16384;           // bytes of a workgroup

template <uint32_t MOVES> struct CopyArgs {
    uint8_t *memory;
    uint64_t page_bytes, layer_bytes;
    uint32_t stretches;                            // of a page
    uint32_t reserved;
    int32_t moves[2 * MOVES];
};

template <uint32_t MOVES> __global__ void __launch_bounds__(256) cache_copy_kernel(const CopyArgs<MOVES> a)
{
    const uint32_t move = blockIdx.x / a.stretches, stretch = blockIdx.x % a.stretches;
    uint8_t *const layer = a.memory + blockIdx.y * a.layer_bytes;
    const uint64_t begin = (uint64_t)stretch * COPY_STRETCH;
    const uint32_t size = (uint32_t)(a.page_bytes - begin < COPY_STRETCH ? a.page_bytes - begin : COPY_STRETCH);
    const uint8_t *from = layer + (uint64_t)a.moves[2 * move] * a.page_bytes + begin;
    uint8_t *to = layer + (uint64_t)a.moves[2 * move + 1] * a.page_bytes + begin;
    u32x4 x[COPY_STRETCH / 4096];
#pragma unroll
    for (uint32_t i = 0; i < COPY_STRETCH / 4096; ++i) {
        const uint32_t at = 4096 * i + 16 * threadIdx.x;
        if (at < size) x[i] = *reinterpret_cast<const u32x4 *>(from + at);
    }
#pragma unroll
    for (uint32_t i = 0; i < COPY_STRETCH / 4096; ++i) {
        const uint32_t at = 4096 * i + 16 * threadIdx.x;
        if (at < size) *reinterpret_cast<u32x4 *>(to + at) = x[i];
    }
}

template <uint32_t MOVES> static mmaemu_status launch_moves(void *memory, const int32_t *moves, uint64_t count, uint64_t page_bytes, uint64_t layers, uint64_t layer_bytes, hipStream_t s)
{
    CopyArgs<MOVES> a;
    a.memory = (uint8_t *)memory;
    a.page_bytes = page_bytes;
    a.layer_bytes = layer_bytes;
    a.stretches = (uint32_t)((page_bytes + COPY_STRETCH - 1) / COPY_STRETCH);
    a.reserved = 0;
    for (uint64_t m = 0; m < count;) {
        // (moves of a page onto itself are left out; a launch's threads count in 32 bits)
        const uint64_t most = (1u << 23) / a.stretches;
        uint32_t n = 0;
        for (; m < count && n < MOVES && n < (most ? most : 1); ++m) {
            if (moves[2 * m] == moves[2 * m + 1]) continue;
            a.moves[2 * n] = moves[2 * m];
            a.moves[2 * n + 1] = moves[2 * m + 1];
            ++n;
        }
        if (!n) break;
        hipLaunchKernelGGL(cache_copy_kernel<MOVES>, dim3(n * a.stretches, (uint32_t)layers), dim3(256), 0, s, a);
        MMAEMU_HIP(hipGetLastError());
    }
    return MMAEMU_OK;
}

mmaemu_status launch_cache_copy(void *memory, const int32_t *moves, uint64_t count, uint64_t page_bytes, uint64_t layers, uint64_t layer_bytes, hipStream_t s)
{
    if (count <= COPY_FEW) return launch_moves<COPY_FEW>(memory, moves, count, page_bytes, layers, layer_bytes, s);
    return launch_moves<COPY_MOVES>(memory, moves, count, page_bytes, layers, layer_bytes, s);
}

} // namespace mmaemu
