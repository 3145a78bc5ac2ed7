// The cache in 4 bits, as memory: pages of a multiple of 32 tokens, in a page each KV head's tokens in granules of 32.  A granule of
// heads of D elements is 34 D bytes: K codes (16 D), V codes (16 D), K scales (D), V scales (D), E2M1 and E8M0 (a scale per 32 elements
// of a token's head).  With the granule's token t = 8 w + 4 a + r (a < 2, r < 4) and element e:
//   K code of e, e + 1:   D 128: a 1024 + e / 32 256 + (4 w + r) 16 + e % 32 / 2          D 64: e / 16 256 + (4 w + r) 16 + a 8 + e % 16 / 2
//   V code of e, e + 1:   D 128: e / 4 % 2 1024 + w 256 + e / 8 16 + e / 2 % 2 8 + t % 8  D 64: w 256 + e / 4 16 + e / 2 % 2 8 + t % 8
//   K scale of block b:   (16 b + 4 w + r) 2 + a          V scale: (w D / 32 + b) 8 + t % 8
// That is what lane 16 g + l of a 16 x 16 x 32 instruction takes, in the lanes' order.  For the scores K is the first operand: lane 16 g + l
// has 16 D / 64 bytes of token 8 (l / 4) + 4 a + l % 4 for instruction row l of half a, so that a lane of the result holds the scores of tokens
// 8 g .. 8 g + 7 (four from each half): with no exchange of lanes these are its eight of the second product's 32.  There V is the first operand: lane
// 16 g + l has tokens 8 g .. + 7 of D / 16 consecutive elements, one of each instruction, so that a lane of the result holds D / 16 consecutive
// outputs.  A byte holds two elements of one token, under one scale: a token is written without reading what is next to it.
//
// Scale codes lie between 104 and 140 (2^-23 .. 2^13), or are 255: every value is an FP16 number, and a BF16 one.
#pragma once
#include "block_scale.hpp"

namespace mmaemu {

constexpr uint32_t CACHE_SCALE_LEAST = 104, CACHE_SCALE_MOST = 140;

struct CacheArgs {
    uint8_t *cache;
    const int32_t *table, *lengths, *begins;
    uint64_t table_stride;
    uint32_t pages, kv_heads, page_granules, sequences, tokens, capacity;      // capacity: tokens that a row of the table holds
};

// One sequence of a call: its tokens are rows `first` .. `first` + n - 1 of the call, the first at position `start` (negative where the
// sequence's length is less than what comes with the call).
struct Sequence { uint32_t first, n; int32_t start, length; };

__device__ __forceinline__ Sequence sequence_of(const CacheArgs &c, uint32_t s)
{
    const int32_t b0 = c.begins[s], b1 = c.begins[s + 1], len = c.lengths[s];
    const uint32_t first = b0 < 0 ? 0u : (uint32_t)b0 > c.tokens ? c.tokens : (uint32_t)b0;
    const uint32_t end = b1 < 0 ? 0u : (uint32_t)b1 > c.tokens ? c.tokens : (uint32_t)b1;
    Sequence q;
    q.first = first;
    q.n = end > first ? end - first : 0u;
    q.length = len < 0 ? 0 : (uint32_t)len > c.capacity ? (int32_t)c.capacity : len;
    q.start = q.length - (int32_t)q.n;
    return q;
}

// a granule of a sequence in a page of the table: NULL where the entry is no page
template <int D> __device__ __forceinline__ uint8_t *granule_at(const CacheArgs &c, int32_t page, uint32_t head, uint32_t granule_of_page)
{
    if ((uint32_t)page >= c.pages) return nullptr;
    return c.cache + ((uint64_t)((uint32_t)page) * c.kv_heads + head) * c.page_granules * (34 * D) + (uint64_t)granule_of_page * (34 * D);
}

mmaemu_status launch_cache_append(const mmaemu_cache_append_fp4_args &a, const CacheArgs &c, hipStream_t s);
mmaemu_status launch_attention_fp4(const mmaemu_attention_fp4_args &a, const CacheArgs &c, hipStream_t s);
uint64_t attention_fp4_workspace(const mmaemu_attention_fp4_args &a);
void attention_fp4_name(const mmaemu_attention_fp4_args &a, char *text, size_t size);
mmaemu_status launch_cache_copy(void *memory, const int32_t *moves, uint64_t count, uint64_t page_bytes, uint64_t layers, uint64_t layer_bytes, hipStream_t s);

} // namespace mmaemu
