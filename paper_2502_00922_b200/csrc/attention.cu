// Attention over the 4-bit cache: one pass over the visible tokens with the running maximum and sum of the softmax.
//
// Scores and sums are products of 16 x 16 codes with eight query rows (rows are query heads that share a key head, of as many tokens as
// there are): mma.sync with the codes as A operand, masked out of the words of a block as they lie (cache_layout.h).  A code c in the low bits
// of a half is the fp16 number c 2^-24, exactly, so nothing is converted.  What the codes stand for, s c + m, comes in around the products:
//   scores   sum_g s_g (c_g . q_g) + sum_g m_g (1 . q_g)     the groups' products apart, times s in fp32; the second sum is one product of its own
//   values   sum_t (p_t s_t,g) c_t + sum_t p_t m_t,g         p_t s_t,g as B operand (one multiplication for two of them a group); the second
//            sum is a product of its own too, and a row of ones in it gives the sum of the p_t
// The tokens are the rows of the first product and the columns of the second: its B operand is the first's result transposed (movmatrix).
//
// Work is cut evenly: the steps of 32 tokens of all (sequence, tile of rows, key head) stand in one line, of which every CTA takes the same
// length; its warps deal the steps of a piece among themselves and add up in shared memory.  Pieces of one line segment that more than one CTA
// works on meet in the workspace, where the last CTA to arrive adds them up in their order.
#include <cuda_runtime.h>

#include "cache_rows.cuh"
#include "decode_common.cuh"
#include "epilogue.cuh"

namespace huffllm {

constexpr uint32_t kStepTokens = 2 * kCacheBlock;
constexpr uint32_t kWaitTries = 1u << 22;

template <int DIM, int NT>
struct AttentionShape {
    static constexpr int kGroups = DIM / 32, kCols = 8 * NT;
    static constexpr int kWarps = DIM * NT <= 128 ? 16 : 8;
    static constexpr int kStages = 2;
    static constexpr uint32_t kBlockBytes = cache_block_bytes(DIM);
    static constexpr uint32_t kRingBytes = kWarps * kStages * 2 * kBlockBytes;
    static constexpr uint32_t kRow = DIM + 4;                    // floats of a column's sums: two of the last four are its reference and weight
    static constexpr uint32_t kMergeBytes = kWarps * kCols * kRow * 4;
    static constexpr uint32_t kSmem = kRingBytes + kMergeBytes;
    static constexpr uint32_t kPartial = kCols * kRow;           // floats of a piece in the workspace
};

// Steps that some row of a sequence sees: the first tokens', then from the window's on.
struct Steps {
    uint32_t sink_end, from, count;                              // step x: x < sink_end ? x : from + x - sink_end
    __device__ __forceinline__ uint32_t step(uint32_t x) const { return x < sink_end ? x : from + x - sink_end; }
};
__device__ __forceinline__ Steps steps_of(const Sequence &S, uint32_t window, uint32_t sinks) {
    Steps s{0, 0, 1};                                            // (rows that see nothing are a step of their own)
    if (S.tokens == 0) return s;
    const uint32_t end = (uint32_t)(S.tokens - 1) / kStepTokens + 1;
    if (window) {
        const int64_t first = (int64_t)S.tokens - S.rows - window + 1;
        if (first > 0) s.from = (uint32_t)(first / kStepTokens);
        const uint32_t seen = min(sinks, (uint32_t)S.tokens);
        s.sink_end = min((seen + kStepTokens - 1) / kStepTokens, s.from);
    }
    s.count = s.sink_end + end - s.from;
    return s;
}

// A stretch of the line: one unit (sequence, key head, tile of rows), its steps x .. end - 1.
struct Walk {
    uint64_t left;                                               // steps of the CTA behind this stretch
    uint32_t b, unit, units, x, end;
    Sequence S;
    Steps steps;
    uint32_t tiles;
    __device__ __forceinline__ void load(const AttentionArgs &A, uint32_t cols) {
        S = sequence_of(A.c, A.starts, A.rows, b);
        steps = steps_of(S, A.window, A.sinks);
        tiles = (S.rows * A.group + cols - 1) / cols;
        units = tiles * A.c.kv_heads;
    }
    // on to the next unit; false at the end of the CTA's line
    __device__ __forceinline__ bool next(const AttentionArgs &A, uint32_t cols) {
        if (left == 0) return false;
        ++unit;
        while (unit >= units) {
            ++b;
            unit = 0;
            load(A, cols);
        }
        x = 0;
        take();
        return true;
    }
    __device__ __forceinline__ void take() {
        const uint32_t room = steps.count - x;
        end = left < room ? x + (uint32_t)left : steps.count;
        left -= end - x;
    }
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t transposed(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *(const uint32_t *)&h;
}
__device__ __forceinline__ uint32_t mul_half2(uint32_t a, uint32_t b) {
    const __half2 h = __hmul2(*(const __half2 *)&a, *(const __half2 *)&b);
    return *(const uint32_t *)&h;
}
__device__ __forceinline__ uint32_t lds32(uint32_t at) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at));
    return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t at) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
    return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
// N consecutive words of shared memory (N * 4-byte aligned for 1, 2, 4)
template <int N>
__device__ __forceinline__ void lds_words(uint32_t at, uint32_t *w) {
    if constexpr (N == 4) {
        const uint4 v = lds128(at);
        w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    } else if constexpr (N == 2) {
        const uint2 v = lds64(at);
        w[0] = v.x, w[1] = v.y;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = lds32(at + 4 * i);
    }
}
__device__ __forceinline__ float low_half(uint32_t w) { return __half2float(__ushort_as_half((uint16_t)w)); }
__device__ __forceinline__ float high_half(uint32_t w) { return __half2float(__ushort_as_half((uint16_t)(w >> 16))); }

template <int DIM, int NT>
__global__ void __launch_bounds__(AttentionShape<DIM, NT>::kWarps * 32, 1) attention_kernel(const __grid_constant__ AttentionArgs A) {
    using Shape = AttentionShape<DIM, NT>;
    constexpr int G = Shape::kGroups, COLS = Shape::kCols, W = Shape::kWarps, STAGES = Shape::kStages, THREADS = W * 32;
    constexpr uint32_t BLOCK = Shape::kBlockBytes, ROW = Shape::kRow;
    constexpr uint32_t kFull = 0xFFFFFFFFu;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t s_bar[W * STAGES];
    __shared__ uint32_t s_here[W * STAGES][2];                   // blocks of a stage that are there
    __shared__ uint64_t s_scan[W + 1], s_found_left;
    __shared__ uint32_t s_found_b, s_last;
    float *const merge = (float *)(smem + Shape::kRingBytes);
    const CacheArgs &C = A.c;
    const uint32_t tid = threadIdx.x, lane = tid % 32, warp = tid / 32, g = lane / 4, t4 = lane % 4;

    if (lane < STAGES) mbar_init(smem_u32(&s_bar[warp * STAGES + lane]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    pdl_launch_dependents();
    pdl_wait_prior_grid();
    if (blockIdx.x == 0) report_faults(C, A.starts, A.rows, A.err);

    // The line: how long it is, and where in it this CTA starts.
    auto weight_of = [&](uint32_t b) -> uint64_t {
        if (b >= C.sequences) return 0;
        const Sequence S = sequence_of(C, A.starts, A.rows, b);
        return (uint64_t)((S.rows * A.group + COLS - 1) / COLS) * C.kv_heads * steps_of(S, A.window, A.sinks).count;
    };
    uint64_t total = 0, mine = weight_of(tid);
    for (uint32_t b0 = 0; b0 < C.sequences; b0 += THREADS) {
        uint64_t w = b0 ? weight_of(b0 + tid) : mine;
        for (int o = 16; o; o >>= 1) w += __shfl_xor_sync(kFull, w, o);
        total += w;
    }
    if (lane == 0) s_scan[warp] = total;
    if (tid == 0) s_found_b = 0, s_found_left = 0;
    __syncthreads();
    total = 0;
    for (int i = 0; i < W; ++i) total += s_scan[i];
    if (total == 0) return;
    // (as many CTAs as find at least a step for every other warp)
    const uint64_t ctas = min((uint64_t)gridDim.x, max((uint64_t)1, (total + W / 2 - 1) / (W / 2)));
    if (blockIdx.x >= ctas) return;
    const uint64_t line_from = blockIdx.x * total / ctas, line_to = (blockIdx.x + 1) * total / ctas;
    uint64_t before = 0;
    for (uint32_t b0 = 0; b0 < C.sequences; b0 += THREADS) {
        const uint64_t w = b0 ? weight_of(b0 + tid) : mine;
        uint64_t sum = w;
        for (int o = 1; o < 32; o <<= 1) {
            const uint64_t up = __shfl_up_sync(kFull, sum, o);
            if (lane >= o) sum += up;
        }
        __syncthreads();
        if (lane == 31) s_scan[warp] = sum;
        __syncthreads();
        uint64_t ahead = before;
        for (uint32_t i = 0; i < W; ++i) {
            if (i < warp) ahead += s_scan[i];
            before += s_scan[i];
        }
        const uint64_t to = ahead + sum, from = to - w;
        if (from <= line_from && line_from < to) s_found_b = b0 + tid, s_found_left = line_from - from;
    }
    __syncthreads();

    Walk ahead;                                                  // the stretch that copies are asked for; `at` is the one worked on
    ahead.b = s_found_b;
    ahead.load(A, COLS);
    ahead.unit = (uint32_t)(s_found_left / ahead.steps.count);
    ahead.x = (uint32_t)(s_found_left % ahead.steps.count);
    ahead.left = line_to - line_from;
    ahead.take();
    Walk at = ahead;
    uint64_t at_first = line_from - at.x;                        // where in the line the unit begins
    bool more = true;
    uint32_t next_x = ahead.x + warp;

    const uint32_t ring = smem_u32(smem) + warp * STAGES * 2 * BLOCK;
    const uint32_t bars = smem_u32(&s_bar[warp * STAGES]);
    // Rows of a unit's tile: positions of its first and last token, and its key head.
    auto tile_of = [&](const Walk &w, int32_t &lo, int32_t &hi) {
        const uint32_t tile = w.unit % w.tiles, r0 = tile * COLS, r1 = min(r0 + COLS, w.S.rows * A.group) - 1;
        const int32_t first = w.S.tokens - (int32_t)w.S.rows;
        lo = first + (int32_t)(r0 / A.group);
        hi = first + (int32_t)(r1 / A.group);
    };
    // Does a row of the tile see one of tokens t .. t + n - 1?
    auto any_seen = [&](uint32_t t, uint32_t n, int32_t lo, int32_t hi) -> bool {
        return (int32_t)t <= hi && (!A.window || (int64_t)t + n > (int64_t)lo - A.window + 1 || t < A.sinks);
    };
    // Ask for the warp's next step.
    auto ask = [&](uint32_t stage) {
        while (more && next_x >= ahead.end) {
            more = ahead.next(A, COLS);
            next_x = ahead.x + warp;
        }
        if (!more) return;
        const uint8_t *src = nullptr;
        if (lane < 2) {
            int32_t lo, hi;
            tile_of(ahead, lo, hi);
            const uint32_t t = ahead.steps.step(next_x) * kStepTokens + lane * kCacheBlock;
            if (any_seen(t, kCacheBlock, lo, hi)) {
                src = block_of(C, ahead.b, t, ahead.unit / ahead.tiles);
                if (!src && A.err) *A.err = (int32_t)ahead.b + 1;
            }
            s_here[warp * STAGES + stage][lane] = src != nullptr;
        }
        const uint32_t count = __popc(__ballot_sync(kFull, src != nullptr));
        if (lane == 0) mbar_expect_tx(bars + 8 * stage, count * BLOCK);
        __syncwarp();
        if (src) bulk_g2s(ring + (stage * 2 + lane) * BLOCK, src, BLOCK, bars + 8 * stage);
        next_x += W;
    };
    __syncwarp();
    for (uint32_t s = 0; s < STAGES; ++s) ask(s);

    uint32_t stage = 0, phase = 0;
    for (bool on = true; on; at_first += at.steps.count, on = at.next(A, COLS)) {
        // ---- the tile's queries, as B operands: column n of a lane is its g, rows its t4's eight channels of a group
        const uint32_t head = at.unit / at.tiles, row0 = at.unit % at.tiles * COLS, rows_all = at.S.rows * A.group;
        uint32_t q[NT][G][4], q_sum[NT][2];
        float factor[NT][2];
        int32_t pos[NT][2];
        int32_t lo, hi;
        tile_of(at, lo, hi);
        const bool wide = !(((uintptr_t)A.q & 15) || A.q_stride % 8);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const uint32_t r = row0 + n * 8 + g, token = r / A.group;
            const uint16_t *src = A.q + (uint64_t)(at.S.first_row + token) * A.q_stride + (uint64_t)(head * A.group + r % A.group) * DIM + t4 * 8;
            uint32_t raw[G][4];
#pragma unroll
            for (int i = 0; i < G; ++i) {
                uint4 v = make_uint4(0, 0, 0, 0);
                if (r < rows_all) {
                    if (wide) {
                        v = __ldcg((const uint4 *)(src + i * 32));
                    } else {
                        uint32_t e[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) e[j] = __ldcg((const unsigned short *)src + i * 32 + j);
                        v = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
                    }
                }
                raw[i][0] = v.x, raw[i][1] = v.y, raw[i][2] = v.z, raw[i][3] = v.w;
            }
            // a row's largest value goes to 2^14 .. 2^15 (by a power of two: exact), so that fp16 holds whatever bf16 does
            auto wide_lo = [&](uint32_t w) { return C.fp16 ? widen16<true>((uint16_t)w) : widen16<false>((uint16_t)w); };
            float most = 0.0f, nan = 0.0f;
#pragma unroll
            for (int i = 0; i < G; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float a = fabsf(wide_lo(raw[i][j])), b = fabsf(wide_lo(raw[i][j] >> 16));
                    most = fmaxf(most, fmaxf(a, b));
                    nan += 0.0f * a + 0.0f * b;
                }
            most = fmaxf(most, __shfl_xor_sync(kFull, most, 1));
            most = fmaxf(most, __shfl_xor_sync(kFull, most, 2));
            nan += __shfl_xor_sync(kFull, nan, 1);
            nan += __shfl_xor_sync(kFull, nan, 2);
            const int shift = max(-90, min(100, 14 - ((int)(__float_as_uint(most) >> 23) - 127)));
            const float up = __uint_as_float((uint32_t)(127 + shift) << 23);
            float sums[G];
#pragma unroll
            for (int i = 0; i < G; ++i) {
                sums[i] = 0.0f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    // (the codes of the second and fourth pair of a word are 16 times as large in their halves)
                    const float a = wide_lo(raw[i][j]) * up, b = wide_lo(raw[i][j] >> 16) * up, down = j & 1 ? 0.0625f : 1.0f;
                    sums[i] += a + b;
                    q[n][i][j] = pack_half2(a * down, b * down);
                }
                sums[i] += __shfl_xor_sync(kFull, sums[i], 1);
                sums[i] += __shfl_xor_sync(kFull, sums[i], 2);
                sums[i] *= 0.03125f;
            }
            // the groups' sums of queries: rows 0..7 of the offsets' B operand their upper halves, 8..15 what these leave
            float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
            for (int i = 0; i < G; i += 2)
                if (t4 * 2 == i) s0 = sums[i], s1 = i + 1 < G ? sums[i + 1] : 0.0f;
            q_sum[n][0] = pack_half2(s0, s1);
            q_sum[n][1] = pack_half2(s0 - low_half(q_sum[n][0]), s1 - high_half(q_sum[n][0]));
            const float f = A.scale * 1.4426950408889634f * __uint_as_float((uint32_t)(127 - shift) << 23) * 16777216.0f + nan;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                factor[n][c] = __shfl_sync(kFull, f, (t4 * 2 + c) * 4);
                const uint32_t rc = row0 + n * 8 + t4 * 2 + c;
                pos[n][c] = rc < rows_all ? at.S.tokens - (int32_t)at.S.rows + (int32_t)(rc / A.group) : -1;
            }
        }

        float acc[NT][2 * G][4], off[NT][4], top[NT][2], ref[NT][2];
        int head_room = 15;                                      // weights are at most 2^head_room: below 2^14 times the largest scale yet
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int j = 0; j < 2 * G; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[n][j][c] = 0.0f;
#pragma unroll
            for (int c = 0; c < 4; ++c) off[n][c] = 0.0f;
            top[n][0] = top[n][1] = ref[n][0] = ref[n][1] = -INFINITY;
        }

        for (uint32_t x = at.x + warp; x < at.end; x += W) {
            {
                uint32_t tries = 0;
                while (!mbar_try_wait(bars + 8 * stage, phase) && ++tries < kWaitTries) {}
                if (tries == kWaitTries && A.err) *A.err = -1;
            }
            const uint32_t base = at.steps.step(x) * kStepTokens, slot = ring + stage * 2 * BLOCK;
            const bool here0 = s_here[warp * STAGES + stage][0], here1 = s_here[warp * STAGES + stage][1];
            if (here0 || here1) {
                // every token of the step seen by every row?
                const bool whole = here0 && here1 && (int32_t)(base + kStepTokens - 1) <= lo &&
                                   (!A.window || (int64_t)base > (int64_t)hi - A.window || base + kStepTokens <= A.sinks);
                float score[2][NT][4];
                uint32_t most2 = 0;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t blk = slot + k * BLOCK;
                    uint32_t wa[G], wb[G], sa[(G + 1) / 2], sb[(G + 1) / 2];
#pragma unroll
                    for (int i = 0; i < G; i += 4) {
                        constexpr int kRest = G % 4 ? G % 4 : 4;
                        if (i + 4 <= G) {
                            lds_words<4>(blk + key_word_at(DIM, 0, i, 0) + lane * 16, wa + i);
                            lds_words<4>(blk + key_word_at(DIM, 0, i, 0) + lane * 16 + 512, wb + i);
                        } else {
                            lds_words<kRest>(blk + key_word_at(DIM, 0, i, 0) + lane * kRest * 4, wa + i);
                            lds_words<kRest>(blk + key_word_at(DIM, 0, i, 0) + lane * kRest * 4 + 128 * kRest, wb + i);
                        }
                    }
                    constexpr int HW = (G + 1) / 2;              // words of a token's scales
                    lds_words<HW>(blk + key_scale_at(DIM, 0, 0) + g * HW * 4, sa);
                    lds_words<HW>(blk + key_scale_at(DIM, 0, 0) + (g + 8) * HW * 4, sb);
                    const uint32_t ma = t4 < HW ? lds32(blk + key_offset_at(DIM, 0, 0) + (g * HW + t4) * 4) : 0u;
                    const uint32_t mb = t4 < HW ? lds32(blk + key_offset_at(DIM, 0, 0) + ((g + 8) * HW + t4) * 4) : 0u;
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        float d[4] = {0, 0, 0, 0};
                        mma_f16_16816(d, ma, mb, ma, mb, q_sum[n][0], q_sum[n][1]);
#pragma unroll
                        for (int c = 0; c < 4; ++c) score[k][n][c] = d[c] * 0x1p-19f;
                    }
#pragma unroll
                    for (int i = 0; i < G; ++i) {
                        const float fa = i & 1 ? high_half(sa[i / 2]) : low_half(sa[i / 2]), fb = i & 1 ? high_half(sb[i / 2]) : low_half(sb[i / 2]);
                        const uint32_t a8 = wa[i] >> 8, b8 = wb[i] >> 8;
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            float d[4] = {0, 0, 0, 0};
                            mma_f16_16816(d, wa[i] & 0x000F000Fu, wb[i] & 0x000F000Fu, wa[i] & 0x00F000F0u, wb[i] & 0x00F000F0u, q[n][i][0], q[n][i][1]);
                            mma_f16_16816(d, a8 & 0x000F000Fu, b8 & 0x000F000Fu, a8 & 0x00F000F0u, b8 & 0x00F000F0u, q[n][i][2], q[n][i][3]);
                            score[k][n][0] = fmaf(d[0], fa, score[k][n][0]);
                            score[k][n][1] = fmaf(d[1], fa, score[k][n][1]);
                            score[k][n][2] = fmaf(d[2], fb, score[k][n][2]);
                            score[k][n][3] = fmaf(d[3], fb, score[k][n][3]);
                        }
                    }
                    // the largest scale of the block's values
#pragma unroll
                    for (int i = 0; i < 8 * G; i += 32) {
                        const uint32_t w = i + lane;
                        uint32_t s2 = w < 8 * G ? lds32(blk + value_scale_at(DIM, 0, 0) + w * 4) : 0u;
                        if (!whole) {                            // (tokens that nobody sees may hold anything)
                            const uint32_t t = base + k * kCacheBlock + w / (2 * G) * 2 + (w & 1) * 8;
                            const bool here = k ? here1 : here0;
                            if (!here || !any_seen(t, 1, lo, hi)) s2 &= 0xFFFF0000u;
                            if (!here || !any_seen(t + 1, 1, lo, hi)) s2 &= 0x0000FFFFu;
                        }
                        const __half2 h = __hmax2(*(const __half2 *)&most2, *(const __half2 *)&s2);
                        most2 = *(const uint32_t *)&h;
                    }
                }
                const uint32_t most = __reduce_max_sync(kFull, max(most2 & 0xFFFFu, most2 >> 16));
                head_room = min(head_room, 28 - (int)(most >> 10));
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float alpha[2];
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float m = -INFINITY;
#pragma unroll
                        for (int k = 0; k < 2; ++k)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                float v = score[k][n][2 * h + c] * factor[n][c];
                                if (!whole) {
                                    const int32_t t = (int32_t)(base + k * kCacheBlock + h * 8 + g);
                                    const bool seen = (k ? here1 : here0) && t <= pos[n][c] &&
                                                      (!A.window || (int64_t)t > (int64_t)pos[n][c] - A.window || (uint32_t)t < A.sinks);
                                    v = seen ? v : -INFINITY;
                                }
                                score[k][n][2 * h + c] = v;
                                m = fmaxf(m, v);
                            }
                        m = fmaxf(m, __shfl_xor_sync(kFull, m, 4));
                        m = fmaxf(m, __shfl_xor_sync(kFull, m, 8));
                        m = fmaxf(m, __shfl_xor_sync(kFull, m, 16));
                        top[n][c] = fmaxf(top[n][c], m);
                        const float r = top[n][c] - (float)head_room;
                        alpha[c] = r == -INFINITY ? 0.0f : ex2(ref[n][c] - r);
                        ref[n][c] = r;
                    }
#pragma unroll
                    for (int j = 0; j < 2 * G; ++j) {
                        acc[n][j][0] *= alpha[0], acc[n][j][1] *= alpha[1];
                        acc[n][j][2] *= alpha[0], acc[n][j][3] *= alpha[1];
                    }
                    off[n][0] *= alpha[0], off[n][1] *= alpha[1], off[n][2] *= alpha[0], off[n][3] *= alpha[1];
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t blk = slot + k * BLOCK;
                    uint32_t p[NT][2];
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const float r0 = ref[n][0] == -INFINITY ? 0.0f : ref[n][0], r1 = ref[n][1] == -INFINITY ? 0.0f : ref[n][1];
                        p[n][0] = transposed(pack_half2(ex2(score[k][n][0] - r0), ex2(score[k][n][1] - r1)));
                        p[n][1] = transposed(pack_half2(ex2(score[k][n][2] - r0), ex2(score[k][n][3] - r1)));
                    }
                    uint2 m = make_uint2(0, 0);
                    if (g < G) m = lds64(blk + value_offset_at(DIM, 0, 0) + (t4 * G + g) * 8);
                    if (!whole) {
                        const bool here = k ? here1 : here0;
                        const uint32_t t = base + k * kCacheBlock + 2 * t4;
                        m.x &= (here && any_seen(t, 1, lo, hi) ? 0xFFFFu : 0u) | (here && any_seen(t + 1, 1, lo, hi) ? 0xFFFF0000u : 0u);
                        m.y &= (here && any_seen(t + 8, 1, lo, hi) ? 0xFFFFu : 0u) | (here && any_seen(t + 9, 1, lo, hi) ? 0xFFFF0000u : 0u);
                    }
                    const uint32_t ones = g == 0 ? 0x3C003C00u : 0u;
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma_f16_16816(off[n], m.x, ones, m.y, ones, p[n][0], p[n][1]);
                    uint32_t w[2 * G];
#pragma unroll
                    for (int j = 0; j < 2 * G; j += 4) {
                        constexpr int kRest = 2 * G % 4 ? 2 : 4;
                        if (j + 4 <= 2 * G) lds_words<4>(blk + value_byte_at(DIM, 0, 16 * j) + lane * 16, w + j);
                        else lds_words<kRest>(blk + value_byte_at(DIM, 0, 16 * j) + lane * kRest * 4, w + j);
                    }
#pragma unroll
                    for (int i = 0; i < G; ++i) {
                        const uint2 s = lds64(blk + value_scale_at(DIM, 0, 0) + (t4 * G + i) * 8);
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            uint32_t p0 = mul_half2(p[n][0], s.x), p1 = mul_half2(p[n][1], s.y);
                            if (!whole) {                        // (what a row does not see is nothing, whatever its scale)
                                p0 &= ((p[n][0] & 0x7FFFu) ? 0xFFFFu : 0u) | ((p[n][0] & 0x7FFF0000u) ? 0xFFFF0000u : 0u);
                                p1 &= ((p[n][1] & 0x7FFFu) ? 0xFFFFu : 0u) | ((p[n][1] & 0x7FFF0000u) ? 0xFFFF0000u : 0u);
                            }
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const uint32_t v = w[2 * i + h], v8 = v >> 8;
                                mma_f16_16816(acc[n][2 * i + h], v & 0x000F000Fu, v & 0x00F000F0u, v8 & 0x000F000Fu, v8 & 0x00F000F0u, p0, p1);
                            }
                        }
                    }
                }
            }
            __syncwarp();
            ask(stage);
            if (++stage == STAGES) stage = 0, phase ^= 1;
        }

        // ---- the warps' sums meet: a column's channels, then its reference and weight
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float *const to = merge + (warp * COLS + n * 8 + 2 * t4 + c) * ROW;
#pragma unroll
                for (int j = 0; j < 2 * G; ++j) {
                    const float m = __shfl_sync(kFull, off[n][c], (j / 2) * 4 + t4);
                    to[16 * j + g] = fmaf(acc[n][j][c], 0x1p24f, m);
                    to[16 * j + 8 + g] = fmaf(acc[n][j][2 + c], 0x1p20f, m);
                }
                if (g == 0) to[DIM] = ref[n][c], to[DIM + 1] = off[n][2 + c];
            }
        __syncthreads();
        const uint32_t n_warps = min((uint32_t)W, at.end - at.x);
        const bool complete = at.x == 0 && at.end == at.steps.count;
        const uint64_t first_cta = ((at_first + 1) * ctas - 1) / total, last_cta = ((at_first + at.steps.count) * ctas - 1) / total;
        float *const piece = A.partials + (2 * (uint64_t)blockIdx.x + (at.x ? 0 : 1)) * Shape::kPartial;
        auto put = [&](uint32_t col, uint32_t d, float value, float weight) {
            const uint32_t r = row0 + col;
            if (r >= rows_all) return;
            const float o = weight == 0.0f ? 0.0f : value / weight;
            A.out[(uint64_t)(at.S.first_row + r / A.group) * A.out_stride + (uint64_t)(head * A.group + r % A.group) * DIM + d] =
                C.fp16 ? round16<true>(o) : round16<false>(o);
        };
        for (uint32_t i = tid; i < COLS * DIM; i += THREADS) {
            const uint32_t col = i / DIM, d = i % DIM;
            float all = -INFINITY, value = 0.0f, weight = 0.0f;
            for (uint32_t w = 0; w < n_warps; ++w) all = fmaxf(all, merge[(w * COLS + col) * ROW + DIM]);
            for (uint32_t w = 0; w < n_warps; ++w) {
                const float *from = merge + (w * COLS + col) * ROW;
                const float scale = from[DIM] == -INFINITY ? (from[DIM + 1] == 0.0f ? 0.0f : NAN) : ex2(from[DIM] - all);
                value = fmaf(scale, from[d], value);
                weight = fmaf(scale, from[DIM + 1], weight);
            }
            if (complete) {
                put(col, d, value, weight);
            } else {
                __stcg(piece + col * ROW + d, value);
                if (d == 0) __stcg(piece + col * ROW + DIM, all), __stcg(piece + col * ROW + DIM + 1, weight);
            }
        }
        __syncthreads();                                         // (the sums are read, the pieces written)
        if (!complete) {
            if (tid == 0) {
                __threadfence();
                const uint32_t count = (uint32_t)(last_cta - first_cta) + 1;
                const bool last = arrive_acq_rel(A.tickets + first_cta) == count - 1;
                if (last) A.tickets[first_cta] = 0;
                __threadfence();
                s_last = last;
            }
            __syncthreads();
            if (s_last) {
                for (uint32_t i = tid; i < COLS * DIM; i += THREADS) {
                    const uint32_t col = i / DIM, d = i % DIM;
                    float all = -INFINITY, value = 0.0f, weight = 0.0f;
                    for (uint64_t c = first_cta; c <= last_cta; ++c)
                        all = fmaxf(all, __ldcg(A.partials + (2 * c + (c == first_cta)) * Shape::kPartial + col * ROW + DIM));
                    for (uint64_t c = first_cta; c <= last_cta; ++c) {
                        const float *from = A.partials + (2 * c + (c == first_cta)) * Shape::kPartial + col * ROW;
                        const float r = __ldcg(from + DIM), l = __ldcg(from + DIM + 1);
                        const float scale = r == -INFINITY ? (l == 0.0f ? 0.0f : NAN) : ex2(r - all);
                        value = fmaf(scale, __ldcg(from + d), value);
                        weight = fmaf(scale, l, weight);
                    }
                    put(col, d, value, weight);
                }
            }
            __syncthreads();
        }
    }
}

template <int DIM, int NT>
static cudaError_t launch_shape(const AttentionArgs &a, uint32_t sms, cudaStream_t stream) {
    using Shape = AttentionShape<DIM, NT>;
    static_assert(Shape::kSmem + 1024 <= 232448, "shared memory of a CTA");
    static_assert(Shape::kPartial <= kAttentionPartial, "a piece's place in the workspace");
    static std::atomic<bool> attr_set[64];   // set twice by racing threads at worst: the call is idempotent
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
        const cudaError_t e = cudaFuncSetAttribute(attention_kernel<DIM, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape::kSmem);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_set[dev].store(true, std::memory_order_release);
    }
    return launch_behind(attention_kernel<DIM, NT>, dim3(sms < kAttentionCtas ? sms : kAttentionCtas), Shape::kWarps * 32, Shape::kSmem, stream, a);
}

// One tile of eight rows where a key head has no more than eight, two where it has (and registers hold them).
cudaError_t launch_attention(const AttentionArgs &a, uint32_t sms, cudaStream_t stream) {
    const bool two = (uint64_t)a.group * ((a.rows + a.c.sequences - 1) / a.c.sequences) > 8;
    switch (a.c.dim) {
        case 64: return two ? launch_shape<64, 2>(a, sms, stream) : launch_shape<64, 1>(a, sms, stream);
        case 96: return two ? launch_shape<96, 2>(a, sms, stream) : launch_shape<96, 1>(a, sms, stream);
        case 128: return two ? launch_shape<128, 2>(a, sms, stream) : launch_shape<128, 1>(a, sms, stream);
        case 192: return launch_shape<192, 1>(a, sms, stream);
        default: return launch_shape<256, 1>(a, sms, stream);
    }
}

}  // namespace huffllm
