// Which token a row of a call is, and where the cache has it.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "cache_layout.h"
#include "decode_step.h"

namespace huffllm {

// Rows, tokens and faults of a sequence, as the device arrays have them.
struct Sequence {
    uint32_t first_row, rows;      // of the call (rows 0 where something is wrong with them)
    int32_t tokens;                // with those rows (0 where the length is no length)
    bool bad;
};
__device__ __forceinline__ Sequence sequence_of(const CacheArgs &c, const int32_t *starts, uint32_t rows, uint32_t b) {
    Sequence s;
    const int32_t n = __ldcg(c.lengths + b);
    const int32_t from = starts ? __ldcg(starts + b) : (int32_t)b, to = starts ? __ldcg(starts + b + 1) : (int32_t)b + 1;
    const bool rows_ok = from >= 0 && to >= from && (uint32_t)to <= rows;
    // (the last 64 numbers are left to sums of positions)
    const bool length_ok = n >= 0 && n <= 0x7FFFFFFF - 64 && (uint64_t)n <= (uint64_t)c.table_stride * c.page_tokens;
    s.first_row = rows_ok ? (uint32_t)from : 0u;
    s.rows = rows_ok ? (uint32_t)(to - from) : 0u;
    s.tokens = length_ok ? n : 0;
    s.bad = !rows_ok || !length_ok;
    return s;
}
// One CTA's look at every sequence: a row finds its own by starts that ascend, and cannot tell where they do not.
__device__ __forceinline__ void report_faults(const CacheArgs &c, const int32_t *starts, uint32_t rows, int32_t *err) {
    if (!err) return;
    for (uint32_t b = threadIdx.x; b < c.sequences; b += blockDim.x)
        if (sequence_of(c, starts, rows, b).bad) *err = (int32_t)b + 1;
}
// The sequence that has row r, if one has: the last one that starts at or in front of it.
__device__ __forceinline__ uint32_t sequence_of_row(const int32_t *starts, uint32_t sequences, uint32_t r) {
    if (!starts) return r;
    uint32_t lo = 0, hi = sequences;                       // starts[lo] <= r or lo == 0; starts[hi] > r or hi == sequences
    while (hi - lo > 1) {
        const uint32_t mid = (lo + hi) / 2;
        if (__ldcg(starts + mid) <= (int32_t)r) lo = mid;
        else hi = mid;
    }
    return lo;
}
// The block that has token `at` of sequence b (key head h), or null where its page is none of the pool's.
__device__ __forceinline__ uint8_t *block_of(const CacheArgs &c, uint32_t b, uint32_t at, uint32_t h) {
    const int32_t page = __ldcg(c.table + (uint64_t)b * c.table_stride + at / c.page_tokens);
    if (page < 0 || (uint32_t)page >= c.pages) return nullptr;
    const uint64_t block = ((uint64_t)page * c.kv_heads + h) * (c.page_tokens / kCacheBlock) + at % c.page_tokens / kCacheBlock;
    return c.pool + block * cache_block_bytes(c.dim);
}

}  // namespace huffllm
