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
// One CTA's look at every sequence: a row finds its own by starts that ascend, and cannot tell where they do not.  (Rows are passed over then; a
// look at all starts by every CTA would cost as many reads as there are sequences and CTAs.)
__device__ __forceinline__ void report_faults(const CacheArgs &c, const int32_t *starts, uint32_t rows, int32_t *err) {
    if (!err) return;
    for (uint32_t b = threadIdx.x; b < c.sequences; b += blockDim.x)
        if (sequence_of(c, starts, rows, b).bad) *err = (int32_t)b + 1;
}
// The sequences that have the rows first + lane (lanes below `rows`, at most 32): the last ones that start at or in front of them.  All lanes of a
// warp; where starts do not ascend, the first sequence that fits.
__device__ __forceinline__ uint32_t sequences_of_rows(const int32_t *starts, uint32_t sequences, uint32_t first, uint32_t rows) {
    constexpr uint32_t kFull = 0xFFFFFFFFu;
    const uint32_t lane = threadIdx.x % 32;
    if (!starts) return min(first + lane, sequences - 1);
    auto run_of = [](uint32_t bits) -> uint32_t { return bits == kFull ? 32 : __ffs(~bits) - 1; };   // (what lies behind a start that is not passed does not count)
    uint32_t lo = 0, hi = sequences;                       // starts[lo] <= first or lo == 0; starts[hi] > first or hi == sequences
    while (hi - lo > 1) {
        const uint32_t step = (hi - lo + 31) / 32, at = lo + lane * step;
        const uint32_t there = __ballot_sync(kFull, lane == 0 || (at < hi && __ldcg(starts + at) <= (int32_t)first));
        const uint32_t k = run_of(there) - 1;
        hi = min(hi, lo + (k + 1) * step);
        lo += k * step;
    }
    if (rows == 1) return lo;
    // the starts behind that one, a lane each: how many are at or in front of a row
    const uint32_t next = lo + 1 + lane;
    const int32_t start = next < sequences ? __ldcg(starts + next) : 0x7FFFFFFF;
    uint32_t mine = lo;
    for (uint32_t r = 1; r < rows; ++r) {
        const uint32_t passed = run_of(__ballot_sync(kFull, start <= (int32_t)(first + r)));
        if (lane == r) mine = lo + passed;
        if (lane == r && passed == 32)                     // (so many sequences without a row)
            while (mine + 1 < sequences && __ldcg(starts + mine + 1) <= (int32_t)(first + r)) ++mine;
    }
    return mine;
}

}  // namespace huffllm
