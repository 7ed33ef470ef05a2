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
// Work is cut evenly: the steps of 32 tokens of all units (sequence, key head, tile of rows) stand in one line, of which every CTA takes the
// same length, and of that every warp.  A warp that has all of a unit writes its output; what warps of one CTA have of a unit meets in shared
// memory, behind the line's end, and what CTAs have of one in the workspace, where the last CTA to arrive adds it up, in the line's order.
// The last warp of a CTA asks for the others' copies (a lane each), two steps ahead of them.
//
// Long lines are bound by memory: 65536 steps of 32 tokens x 128 channels more (335 MB) take 55 us more, 6.1 TB/s, 0.93 of the measured copy rate.  Some
// 17 us are a launch's own: 5 to 6 before the first sums (lengths, page, block and queries come one behind the other), 5 to 8 for joining, the rest
// warps that end at different times.  40 sequences of up to 8192 tokens, 64 heads over 8: 60 us, 4.3 TB/s; one of 4096, 32 over 8: 12.4 us.
// Tiles of sixteen rows (pieces of prompts) are bound by the issue of what surrounds the matrix instructions (500 instructions a step, of which 72 are those).
#include <cuda_runtime.h>
#include <cfloat>

#include "cache_rows.cuh"
#include "decode_common.cuh"
#include "epilogue.cuh"

namespace huffllm {

constexpr uint32_t kStepTokens = 2 * kCacheBlock;
constexpr uint32_t kLead = 1;                     // steps that a unit's beginning takes as long as (its queries, its sums): they count in the line
// A wait gives up after about a second: so many tries of one that sleeps for some microseconds, and of one that does not.
constexpr uint32_t kWaitTries = 1u << 17, kPollTries = 1u << 25;
constexpr int kSlack = 4;                        // a weight's exponent is set this far below its cap, so that few later ones are above it

// As many warps as registers and shared memory hold: 128 registers a thread where a lane's sums are 32 (sixteen warps), 255 where they are 64 (eight; with
// 186 registers and eleven warps the sums spill: pieces of 48 tokens over 2000 in an 8B-shaped layer 64 us instead of 54).  Measured at 128 channels; 64
// channels with sixteen rows spill 230 bytes at 128 registers.
template <int DIM, int NT>
struct AttentionShape {
    static constexpr int kGroups = DIM / 32, kCols = 8 * NT;
    static constexpr int kWarps = DIM * NT <= 128 ? 15 : 7;      // that compute; one more asks for their copies
    static constexpr int kStages = DIM * NT == 256 && DIM == 128 ? 3 : 2;
    static constexpr uint32_t kBlockBytes = cache_block_bytes(DIM);
    static constexpr uint32_t kRingBytes = kWarps * kStages * 2 * kBlockBytes;
    static constexpr uint32_t kRow = DIM + 4;                    // floats of a column's sums: two of the last four are its reference and weight
    static constexpr uint32_t kPiece = kCols * kRow;             // floats of what is known of a unit
    static constexpr uint32_t kSmem = kRingBytes + kWarps * kPiece * 4;
    static_assert(kStages * 2 * kBlockBytes >= kPiece * 4, "a warp's last piece lies where its copies did");
};

// Steps that some row of a sequence sees: the first tokens', then from the window's on.
struct Steps {
    uint32_t sink_end, from, count;                              // the first kLead of the `count` are none
    __device__ __forceinline__ uint32_t step(uint32_t x) const { return x - kLead < sink_end ? x - kLead : from + x - kLead - sink_end; }
};
__device__ __forceinline__ Steps steps_of(const Sequence &S, uint32_t window, uint32_t sinks) {
    Steps s{0, 0, kLead + 1};                                    // (rows that see nothing are a step of their own)
    if (S.tokens == 0) return s;
    const uint32_t end = (uint32_t)(S.tokens - 1) / kStepTokens + 1;
    if (window) {
        const int64_t first = (int64_t)S.tokens - S.rows - window + 1;
        if (first > 0) s.from = (uint32_t)first / kStepTokens;
        const uint32_t seen = min(sinks, (uint32_t)S.tokens);
        s.sink_end = min((seen + kStepTokens - 1) / kStepTokens, s.from);
    }
    s.count = kLead + s.sink_end + end - s.from;
    return s;
}

// What is known of a unit that a warp had a part of.
struct Piece {
    uint64_t begin;                                              // where in the line the unit begins
    uint32_t count;                                              // its steps (0: no piece)
    uint32_t first_row, rows, head, row0;                        // of the sequence: its first row, all its rows times heads; of the unit: key head, first row
};
// A stretch of the line: one unit (sequence, key head, tile of rows), its steps x .. end - 1.
struct Walk {
    uint64_t left;                                               // steps of the warp behind this stretch
    uint32_t b, unit, units, x, end, tiles;
    uint32_t head, row0;                                         // of the unit: key head, first row of the tile
    int32_t lo, hi, from;                                        // tokens of the tile's first and last row; the first one that the first row's window has
    Sequence S;
    Steps steps;
    __device__ __forceinline__ void load(const AttentionArgs &A, uint32_t cols) {
        S = sequence_of(A.c, A.starts, A.rows, b);
        know(A, cols);
    }
    __device__ __forceinline__ void know(const AttentionArgs &A, uint32_t cols) {
        steps = steps_of(S, A.window, A.sinks);
        tiles = (S.rows * A.group + cols - 1) / cols;
        units = tiles * A.c.kv_heads;
    }
    __device__ __forceinline__ void take(const AttentionArgs &A, uint32_t cols) {
        head = unit / tiles;
        row0 = unit % tiles * cols;
        const int32_t first = S.tokens - (int32_t)S.rows;
        lo = first + (int32_t)(row0 / A.group);
        hi = first + (int32_t)((min(row0 + cols, S.rows * A.group) - 1) / A.group);
        from = first_seen(A, lo);
        const uint32_t room = steps.count - x;
        end = left < room ? x + (uint32_t)left : steps.count;
        left -= end - x;
    }
    // on to the next unit; false at the end of the warp's line
    __device__ __forceinline__ bool next(const AttentionArgs &A, uint32_t cols) {
        if (left == 0) return false;
        ++unit;
        while (unit >= units) {
            ++b;
            unit = 0;
            load(A, cols);
        }
        x = 0;
        take(A, cols);
        return true;
    }
    static __device__ __forceinline__ int32_t first_seen(const AttentionArgs &A, int32_t pos) {
        return A.window && (int64_t)pos >= (int64_t)A.window ? pos - (int32_t)A.window + 1 : 0;
    }
    // does some row of the tile see one of the tokens t .. t + n - 1?
    __device__ __forceinline__ bool any_seen(const AttentionArgs &A, uint32_t t, uint32_t n) const {
        return (int32_t)t <= hi && ((int32_t)(t + n) > from || t < A.sinks);
    }
    // does every row see all tokens of the step from t on?
    __device__ __forceinline__ bool all_seen(const AttentionArgs &A, uint32_t t) const {
        return (int32_t)(t + kStepTokens) <= lo + 1 && ((int32_t)t >= first_seen(A, hi) || t + kStepTokens <= A.sinks);
    }
};

// (a division of 64 bits is some hundred instructions, and hardly a line is that long)
__device__ __forceinline__ uint64_t quotient(uint64_t a, uint64_t b) { return (a | b) >> 32 ? a / b : (uint32_t)a / (uint32_t)b; }
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
// What the product (a + rest) * s leaves beyond `product`, the rounded a * s.
__device__ __forceinline__ uint32_t rest_half2(uint32_t a, uint32_t rest, uint32_t s, uint32_t product) {
    const __half2 scale = *(const __half2 *)&s, left = __hfma2(*(const __half2 *)&a, scale, __hneg2(*(const __half2 *)&product));
    const __half2 h = __hfma2(*(const __half2 *)&rest, scale, left);
    return *(const uint32_t *)&h;
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

// Products alone, without a sum to add them to
__device__ __forceinline__ void mma_f16_16816_new(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ void sts32(uint32_t at, uint32_t v) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory"); }

// FINE: for results in FP16, which show what rounding p_t and p_t s_t,g to 11 bits costs (twice the error of the results' own rounding): both keep
// what they leave, as a second number of 11 bits, exactly, and the products with values are taken twice.  (A seventh more instructions.)  Results in BF16
// have one of 11 bits: with both, 40 sequences of up to 8192 tokens take 66 us instead of 60, pieces of prompts 63 instead of 54, and the error against
// 64 bits, 1.7e-3 of the values, is that of rounding the results either way.
template <int DIM, int NT, bool FINE>
__global__ void __launch_bounds__(AttentionShape<DIM, NT>::kWarps * 32 + 32, 1) attention_kernel(const __grid_constant__ AttentionArgs A) {
    using Shape = AttentionShape<DIM, NT>;
    constexpr int G = Shape::kGroups, COLS = Shape::kCols, W = Shape::kWarps, STAGES = Shape::kStages, THREADS = W * 32 + 32;
    constexpr uint32_t BLOCK = Shape::kBlockBytes, ROW = Shape::kRow;
    constexpr uint32_t kFull = 0xFFFFFFFFu;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t s_bar[2][W * STAGES];      // a stage's copies have arrived; a stage has been read
    __shared__ uint64_t s_start[W];                              // where in the line the first sequence of a warp begins
    __shared__ uint32_t s_start_b[W];                            // ... and which one it is
    __shared__ Sequence s_start_s[W];
    __shared__ uint32_t s_here[W * STAGES][2];                   // blocks of a stage that are there
    __shared__ Piece s_piece[W][2];
    __shared__ uint32_t s_late[W];                               // a wait of the warp that gave up: 1 + 2 * stage + phase
    __shared__ uint2 s_join[2];                                  // units that this CTA is the last to arrive at: first CTA and number of pieces
    float *const first_pieces = (float *)(smem + Shape::kRingBytes);
    auto piece_at = [&](uint32_t w, uint32_t which) { return which ? (float *)(smem + w * STAGES * 2 * BLOCK) : first_pieces + w * Shape::kPiece; };
    const CacheArgs &C = A.c;
    const uint32_t tid = threadIdx.x, lane = tid % 32, warp = tid / 32, g = lane / 4, t4 = lane % 4;

    if (warp < W && lane < STAGES) mbar_init(smem_u32(&s_bar[0][warp * STAGES + lane]), 1), mbar_init(smem_u32(&s_bar[1][warp * STAGES + lane]), 1);
    if (warp < W && lane < 2) s_piece[warp][lane].count = 0, s_late[warp] = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    pdl_launch_dependents();
    pdl_wait_prior_grid();

    // The line: how long it is, and where in it this CTA starts (every warp finds out by itself).
    Sequence seen;                                               // the last one that was weighed
    auto weight_of = [&](uint32_t b) -> uint64_t {
        if (b >= C.sequences) return 0;
        const Sequence &S = seen;
        seen = sequence_of(C, A.starts, A.rows, b);
        if (S.bad && tid < 32 && blockIdx.x == 0 && A.err) *A.err = (int32_t)b + 1;
        return (uint64_t)((S.rows * A.group + COLS - 1) / COLS) * C.kv_heads * steps_of(S, A.window, A.sinks).count;
    };
    const uint64_t first = weight_of(lane);
    const Sequence first_seen = seen;
    uint64_t total = first;
    for (uint32_t b0 = 32; b0 < C.sequences; b0 += 32) total += weight_of(b0 + lane);
    for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(kFull, total, o);
    if (total == 0) return;
    // (as many CTAs as find at least a step for every other of their warps)
    const uint32_t ctas = (uint32_t)min((uint64_t)gridDim.x, (total + W / 2 - 1) / (W / 2));
    if (blockIdx.x >= ctas) return;
    const uint64_t cta_each = quotient(total, ctas), cta_rest = total - cta_each * ctas;       // (the first cta_rest CTAs have a step more)
    const uint64_t cta_from = cta_each * blockIdx.x + min((uint64_t)blockIdx.x, cta_rest), cta_to = cta_from + cta_each + (blockIdx.x < cta_rest ? 1 : 0);
    auto cta_of = [&](uint64_t step) -> uint32_t {
        const uint64_t longer = cta_rest * (cta_each + 1);
        return (uint32_t)(step < longer ? quotient(step, cta_each + 1) : cta_rest + quotient(step - longer, cta_each));
    };
    // (warps without a step are the last ones: a unit's pieces are those of warps that follow each other)
    const uint64_t each = (cta_to - cta_from) / W, rest = (cta_to - cta_from) % W;
    const uint32_t reader = warp < W ? warp : min(lane, W - 1);  // the last warp's lanes ask for a warp's copies each
    const uint64_t line_from = cta_from + each * reader + min((uint64_t)reader, rest), line_to = line_from + each + (reader < rest ? 1 : 0);
    if (warp < W && line_from < line_to) {
        uint64_t before = 0;
        for (uint32_t b0 = 0;; b0 += 32) {
            const uint64_t w = b0 ? weight_of(b0 + lane) : first;
            uint64_t sum = w;
            for (int o = 1; o < 32; o <<= 1) {
                const uint64_t up = __shfl_up_sync(kFull, sum, o);
                if (lane >= o) sum += up;
            }
            const uint32_t behind = __ballot_sync(kFull, before + sum > line_from);
            if (behind) {                                        // (there is one: the line goes on behind its start)
                const int k = __ffs(behind) - 1;
                before += __shfl_sync(kFull, sum - w, k);
                if (lane == k) s_start_b[warp] = b0 + k, s_start_s[warp] = b0 ? seen : first_seen;
                if (lane == 0) s_start[warp] = before;
                break;
            }
            before += __shfl_sync(kFull, sum, 31);
        }
    }
    __syncthreads();
    const uint32_t ring = smem_u32(smem) + reader * STAGES * 2 * BLOCK;
    const uint32_t bars = smem_u32(&s_bar[0][reader * STAGES]), read_bars = smem_u32(&s_bar[1][reader * STAGES]);
    Walk at;
    if (line_from < line_to) {
        at.b = s_start_b[reader];
        at.S = s_start_s[reader];
        at.know(A, COLS);
        const uint64_t in = line_from - s_start[reader];
        at.unit = (uint32_t)quotient(in, at.steps.count);
        at.x = (uint32_t)(in - (uint64_t)at.unit * at.steps.count);
        at.left = line_to - line_from;
        at.take(A, COLS);
    }
    if (warp == W) {
        // The copies: a lane looks up its warp's next pages, and asks for them as soon as their stage has been read.
        const uint32_t page_blocks = C.page_tokens / kCacheBlock;
        bool more = lane < W && line_from < line_to;
        uint32_t x = more ? max(at.x, kLead) : 0, stage = 0, phase = 1, in_page[2] = {0, 0};   // (a fresh barrier's phase in front of its first is over)
        int32_t page[2] = {-1, -1};
        bool wanted[2] = {false, false};
        auto look_up = [&]() {
            while (x >= at.end) {
                more = at.next(A, COLS);
                x = kLead;
                if (!more) return;
            }
            const uint32_t block = at.steps.step(x) * 2;
            uint32_t i = __umulhi(block, A.page_recip);          // block / page_blocks, or one less
            in_page[0] = block - i * page_blocks;
            if (in_page[0] >= page_blocks) ++i, in_page[0] -= page_blocks;
            const int32_t *const entry = C.table + (uint64_t)at.b * C.table_stride + i;
            const bool turns = in_page[0] + 1 == page_blocks;
            in_page[1] = turns ? 0 : in_page[0] + 1;
            wanted[0] = at.any_seen(A, block * kCacheBlock, kCacheBlock);
            wanted[1] = at.any_seen(A, block * kCacheBlock + kCacheBlock, kCacheBlock);
            if (wanted[0] || (wanted[1] && !turns)) page[0] = __ldcg(entry);
            if (wanted[1] && turns) page[1] = __ldcg(entry + 1);
            else page[1] = page[0];
        };
        if (more) look_up();
        for (uint32_t tries = 0; __any_sync(kFull, more) && tries < kPollTries; ++tries) {
            const bool ready = more && mbar_test_wait(read_bars + 8 * stage, phase);
            if (__any_sync(kFull, ready)) tries = 0;
            if (ready) {
                bool here[2];
                const uint8_t *src[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    here[k] = wanted[k] && page[k] >= 0 && (uint32_t)page[k] < C.pages;
                    if (wanted[k] && !here[k] && A.err) *A.err = (int32_t)at.b + 1;
                    src[k] = C.pool + (((uint64_t)(uint32_t)page[k] * C.kv_heads + at.head) * page_blocks + in_page[k]) * BLOCK;
                    s_here[reader * STAGES + stage][k] = here[k];
                }
                mbar_expect_tx(bars + 8 * stage, (here[0] + here[1]) * BLOCK);
                const uint32_t to = ring + stage * 2 * BLOCK;
                if (here[0] && here[1] && src[1] == src[0] + BLOCK) {
                    bulk_g2s(to, src[0], 2 * BLOCK, bars + 8 * stage);
                } else {
                    if (here[0]) bulk_g2s(to, src[0], BLOCK, bars + 8 * stage);
                    if (here[1]) bulk_g2s(to + BLOCK, src[1], BLOCK, bars + 8 * stage);
                }
                if (++stage == STAGES) stage = 0, phase ^= 1;
                ++x;
                look_up();
            }
        }
        if (more && A.err) *A.err = -1;
    } else if (line_from < line_to) {
    uint64_t at_first = line_from - at.x;                        // where in the line the unit begins
    uint32_t stage = 0, phase = 0;
    for (bool on = true; on; at_first += at.steps.count, on = at.next(A, COLS)) {
        // ---- the tile's queries, as B operands: column n of a lane is its g, rows its t4's eight channels of a group
        const uint32_t head = at.head, row0 = at.row0, rows_all = at.S.rows * A.group;
        uint32_t q[NT][G][4], q_sum[NT][2];
        float factor[NT][2];
        int32_t pos[NT][2];
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
            float most = 0.0f, nan = 0.0f * A.scale;
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
            const int shift = max(14 - 127, min(100, 14 - ((int)(__float_as_uint(most) >> 23) - 127)));
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
            // (beyond fp32, which takes queries of 2^120 or so, the largest number does as well: scores that differ at all are then 2^50 apart, or more)
            const float f = fminf(fmaxf(A.scale * 1.4426950408889634f * __uint_as_float((uint32_t)(127 - shift) << 23) * 16777216.0f, -FLT_MAX), FLT_MAX) + nan;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                factor[n][c] = __shfl_sync(kFull, f, (t4 * 2 + c) * 4);
                const uint32_t rc = row0 + n * 8 + t4 * 2 + c;
                pos[n][c] = rc < rows_all ? at.S.tokens - (int32_t)at.S.rows + (int32_t)(rc / A.group) : -1;
            }
        }

        float acc[NT][2 * G][4], off[NT][4], ref[NT][2];         // weights are 2^(score - ref)
        float cap[NT][2];                                        // ... of at most 2^cap (minus infinity: the row has not seen a token yet)
        int room = 15;                                           // the next cap: 2^room times the largest scale of the values yet is below 2^14
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int j = 0; j < 2 * G; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[n][j][c] = 0.0f;
#pragma unroll
            for (int c = 0; c < 4; ++c) off[n][c] = 0.0f;
            ref[n][0] = ref[n][1] = 0.0f;
            cap[n][0] = cap[n][1] = -INFINITY;
        }

        for (uint32_t x = max(at.x, kLead); x < at.end; ++x) {
            {
                uint32_t tries = 0;
                while (!mbar_try_wait(bars + 8 * stage, phase) && ++tries < kWaitTries) {}
                if (tries == kWaitTries) {
                    s_late[warp] = 1 + 2 * stage + phase;
                    if (A.err) *A.err = -1;
                }
            }
            const uint32_t base = at.steps.step(x) * kStepTokens, slot = ring + stage * 2 * BLOCK;
            const bool here0 = s_here[warp * STAGES + stage][0], here1 = s_here[warp * STAGES + stage][1];
            if (here0 || here1) {
                const bool whole = here0 && here1 && at.all_seen(A, base);
                if (!whole) {
                    // what nobody sees may hold anything: its scales and offsets of values become 0, its scores (below) minus infinity
#pragma unroll 1
                    for (uint32_t w = lane; w < 16 * G; w += 32) {
                        const uint32_t k = w / (8 * G), i = w % (8 * G), t = base + k * kCacheBlock + i / (2 * G) * 2 + (i & 1) * 8;
                        const bool here = k ? here1 : here0;
                        const uint32_t mask = (here && at.any_seen(A, t, 1) ? 0xFFFFu : 0u) | (here && at.any_seen(A, t + 1, 1) ? 0xFFFF0000u : 0u);
                        const uint32_t s_at = slot + k * BLOCK + value_scale_at(DIM, 0, 0) + i * 4, m_at = slot + k * BLOCK + value_offset_at(DIM, 0, 0) + i * 4;
                        sts32(s_at, lds32(s_at) & mask);
                        sts32(m_at, lds32(m_at) & mask);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                }
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
                        float d[4];
                        mma_f16_16816_new(d, ma, mb, ma, mb, q_sum[n][0], q_sum[n][1]);
#pragma unroll
                        for (int c = 0; c < 4; ++c) score[k][n][c] = d[c] * 0x1p-19f;
                    }
#pragma unroll
                    for (int i = 0; i < G; ++i) {
                        const float fa = i & 1 ? high_half(sa[i / 2]) : low_half(sa[i / 2]), fb = i & 1 ? high_half(sb[i / 2]) : low_half(sb[i / 2]);
                        const uint32_t a8 = wa[i] >> 8, b8 = wb[i] >> 8;
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            float d[4];
                            mma_f16_16816_new(d, wa[i] & 0x000F000Fu, wb[i] & 0x000F000Fu, wa[i] & 0x00F000F0u, wb[i] & 0x00F000F0u, q[n][i][0], q[n][i][1]);
                            mma_f16_16816(d, a8 & 0x000F000Fu, b8 & 0x000F000Fu, a8 & 0x00F000F0u, b8 & 0x00F000F0u, q[n][i][2], q[n][i][3]);
                            score[k][n][0] = fmaf(d[0], fa, score[k][n][0]);
                            score[k][n][1] = fmaf(d[1], fa, score[k][n][1]);
                            score[k][n][2] = fmaf(d[2], fb, score[k][n][2]);
                            score[k][n][3] = fmaf(d[3], fb, score[k][n][3]);
                        }
                    }
                    // the largest scale of the block's values (as whole numbers: they are not negative, and a NaN is larger than any)
#pragma unroll
                    for (int i = 0; i < 8 * G; i += 32)
                        if (8 * G % 32 == 0 || i + lane < 8 * G) most2 = __vmaxu2(most2, lds32(blk + value_scale_at(DIM, 0, 0) + (i + lane) * 4));
                }
                // to exponents of the weights
                bool over = (max(most2 & 0xFFFFu, most2 >> 16) >> 10) > (uint32_t)(28 - room);
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int c = 0; c < 4; ++c) score[k][n][c] = fmaf(score[k][n][c], factor[n][c & 1], -ref[n][c & 1]);
                if (!whole) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const int32_t seen_from = Walk::first_seen(A, pos[n][c]);
#pragma unroll
                            for (int k = 0; k < 2; ++k)
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    const int32_t t = (int32_t)(base + k * kCacheBlock + h * 8 + g);
                                    const bool seen = (k ? here1 : here0) && t <= pos[n][c] && (t >= seen_from || (uint32_t)t < A.sinks);
                                    if (!seen) score[k][n][2 * h + c] = -INFINITY;
                                }
                        }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        over = over || fmaxf(fmaxf(score[0][n][c], score[0][n][2 + c]), fmaxf(score[1][n][c], score[1][n][2 + c])) > cap[n][c];
                if (__any_sync(kFull, over)) {
                    // weights too large for what they are relative to, the first that a row sees, or scales larger than any yet
                    uint32_t most = __reduce_max_sync(kFull, max(most2 & 0xFFFFu, most2 >> 16));
                    if (most >= 0x7C00u) {
                        // groups of values that stand for NaN: the rows that see one get it by way of the offsets, and its scale becomes 0
                        most = 0;
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const uint32_t scales = slot + k * BLOCK + value_scale_at(DIM, 0, 0);
                            uint2 s = make_uint2(0, 0);
                            if (g < G) s = lds64(scales + (t4 * G + g) * 8);
                            auto nans = [](uint32_t h2) { return ((h2 & 0x7FFFu) > 0x7C00u ? 0x3C00u : 0u) | ((h2 & 0x7FFF0000u) > 0x7C000000u ? 0x3C000000u : 0u); };
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                auto seen = [&](int c) { return score[k][n][c] > -INFINITY ? 1.0f : 0.0f; };
                                const uint32_t b0 = transposed(pack_half2(seen(0), seen(1))), b1 = transposed(pack_half2(seen(2), seen(3)));
                                float d[4];
                                mma_f16_16816_new(d, nans(s.x), 0u, nans(s.y), 0u, b0, b1);
                                off[n][0] = d[0] > 0.0f ? NAN : off[n][0];
                                off[n][1] = d[1] > 0.0f ? NAN : off[n][1];
                            }
                            __syncwarp();
#pragma unroll 1
                            for (uint32_t w = lane; w < 8 * G; w += 32) {
                                uint32_t h2 = lds32(scales + w * 4);
                                h2 &= ((h2 & 0x7FFFu) > 0x7C00u ? 0u : 0xFFFFu) | ((h2 & 0x7FFF0000u) > 0x7C000000u ? 0u : 0xFFFF0000u);
                                sts32(scales + w * 4, h2);
                                most = max(most, max(h2 & 0xFFFFu, h2 >> 16));
                            }
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                        most = __reduce_max_sync(kFull, most);
                    }
                    room = min(room, 28 - (int)(most >> 10));
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        float alpha[2];
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            float m = fmaxf(fmaxf(score[0][n][c], score[0][n][2 + c]), fmaxf(score[1][n][c], score[1][n][2 + c]));
                            m = fmaxf(m, __shfl_xor_sync(kFull, m, 4));
                            m = fmaxf(m, __shfl_xor_sync(kFull, m, 8));
                            m = fmaxf(m, __shfl_xor_sync(kFull, m, 16));
                            const bool none = cap[n][c] == -INFINITY;        // (nothing seen yet)
                            float by = 0.0f;
                            if (m > fminf(cap[n][c], (float)room)) by = m - (float)(room - kSlack);
                            alpha[c] = none ? 0.0f : ex2(-by);
                            ref[n][c] += by;
#pragma unroll
                            for (int k = 0; k < 2; ++k) score[k][n][c] -= by, score[k][n][2 + c] -= by;
                            if (!none || m > -INFINITY) cap[n][c] = (float)room;
                        }
#pragma unroll
                        for (int j = 0; j < 2 * G; ++j) {
                            acc[n][j][0] *= alpha[0], acc[n][j][1] *= alpha[1];
                            acc[n][j][2] *= alpha[0], acc[n][j][3] *= alpha[1];
                        }
                        off[n][0] *= alpha[0], off[n][1] *= alpha[1], off[n][2] *= alpha[0], off[n][3] *= alpha[1];
                    }
                }
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const uint32_t blk = slot + k * BLOCK;
                    uint32_t p[NT][2], rest[NT][2];
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float e0 = ex2(score[k][n][2 * h]), e1 = ex2(score[k][n][2 * h + 1]);
                            const uint32_t both = pack_half2(e0, e1);
                            p[n][h] = transposed(both);
                            if (FINE) rest[n][h] = transposed(pack_half2(e0 - low_half(both), e1 - high_half(both)));
                        }
                    uint2 m = make_uint2(0, 0);
                    if (g < G) m = lds64(blk + value_offset_at(DIM, 0, 0) + (t4 * G + g) * 8);
                    const uint32_t ones = g == 0 ? 0x3C003C00u : 0u;
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        mma_f16_16816(off[n], m.x, ones, m.y, ones, p[n][0], p[n][1]);
                        if (FINE) mma_f16_16816(off[n], m.x, ones, m.y, ones, rest[n][0], rest[n][1]);
                    }
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
                            const uint32_t p0 = mul_half2(p[n][0], s.x), p1 = mul_half2(p[n][1], s.y);
                            const uint32_t r0 = FINE ? rest_half2(p[n][0], rest[n][0], s.x, p0) : 0u, r1 = FINE ? rest_half2(p[n][1], rest[n][1], s.y, p1) : 0u;
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const uint32_t v = w[2 * i + h], v8 = v >> 8;
                                mma_f16_16816(acc[n][2 * i + h], v & 0x000F000Fu, v & 0x00F000F0u, v8 & 0x000F000Fu, v8 & 0x00F000F0u, p0, p1);
                                if (FINE) mma_f16_16816(acc[n][2 * i + h], v & 0x000F000Fu, v & 0x00F000F0u, v8 & 0x000F000Fu, v8 & 0x00F000F0u, r0, r1);
                            }
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(read_bars + 8 * stage);
            if (++stage == STAGES) stage = 0, phase ^= 1;
        }

        // ---- the unit's channels; a column's reference (minus infinity: nothing seen) and weight
        if (at.x == 0 && at.end == at.steps.count) {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                float by[2];
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const float weight = __shfl_sync(kFull, off[n][2 + c], t4);
                    by[c] = weight == 0.0f ? 0.0f : 1.0f / weight;
                }
                const uint32_t r = row0 + n * 8 + g;             // (behind the transposition a lane has one row, two channels)
                uint16_t *const to = A.out + (uint64_t)(at.S.first_row + r / A.group) * A.out_stride + (uint64_t)(head * A.group + r % A.group) * DIM + 2 * t4;
                const bool in = r < rows_all, paired = ((uintptr_t)to & 3) == 0;
#pragma unroll
                for (int j = 0; j < 2 * G; ++j) {
                    const float m0 = __shfl_sync(kFull, off[n][0], (j / 2) * 4 + t4), m1 = __shfl_sync(kFull, off[n][1], (j / 2) * 4 + t4);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float up = h ? 0x1p20f : 0x1p24f;
                        float o0 = fmaf(acc[n][j][2 * h], up, m0) * by[0], o1 = fmaf(acc[n][j][2 * h + 1], up, m1) * by[1];
                        const uint32_t v = transposed(C.fp16 ? round16<true>(o0) | (uint32_t)round16<true>(o1) << 16
                                                             : round16<false>(o0) | (uint32_t)round16<false>(o1) << 16);
                        uint16_t *const o = to + 16 * j + 8 * h;
                        if (in && paired) *(uint32_t *)o = v;
                        else if (in) o[0] = (uint16_t)v, o[1] = (uint16_t)(v >> 16);
                    }
                }
            }
        } else {
            const uint32_t which = at.x ? 0 : 1;
            float *const piece = piece_at(warp, which);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float *const to = piece + (n * 8 + 2 * t4 + c) * ROW;
#pragma unroll
                    for (int j = 0; j < 2 * G; ++j) {
                        const float m = __shfl_sync(kFull, off[n][c], (j / 2) * 4 + t4);
                        to[16 * j + g] = fmaf(acc[n][j][c], 0x1p24f, m);
                        to[16 * j + 8 + g] = fmaf(acc[n][j][2 + c], 0x1p20f, m);
                    }
                    if (g == 0) *(float2 *)(to + DIM) = make_float2(cap[n][c] == -INFINITY ? -INFINITY : ref[n][c], off[n][2 + c]);
                }
            if (lane == 0) s_piece[warp][which] = Piece{at_first, at.steps.count, at.S.first_row, rows_all, head, row0};
        }
    }
    // (what is late may still land: the CTA's memory stays its own for another wait)
    if (const uint32_t late = s_late[warp])
        for (uint32_t tries = 0; !mbar_try_wait(bars + 8 * ((late - 1) / 2), (late - 1) % 2) && tries < kWaitTries; ++tries) {}
    }
    __syncthreads();

    // ---- units of which more than one warp has a piece: a run of pieces in the order of the line
    // Joins four channels of one column of `count` pieces: `load(i, value, tail)` brings a piece's sums, and their reference and weight.  `batch`
    // pieces are on their way together.
    auto join = [&](auto batch, uint32_t count, auto load, float4 &value, float2 &tail) {
        constexpr uint32_t N = decltype(batch)::value;
        value = make_float4(0, 0, 0, 0);
        tail = make_float2(-INFINITY, 0.0f);
        for (uint32_t base = 0; base < count; base += N) {
            float4 v[N];
            float2 t[N];
#pragma unroll
            for (uint32_t i = 0; i < N; ++i) {
                v[i] = make_float4(0, 0, 0, 0), t[i] = make_float2(-INFINITY, 0.0f);
                if (base + i < count) load(base + i, v[i], t[i]);
            }
            float top = tail.x;
#pragma unroll
            for (uint32_t i = 0; i < N; ++i) top = fmaxf(top, t[i].x);
            auto scale_of = [&](float2 from) { return from.x == -INFINITY ? (from.y == 0.0f ? 0.0f : NAN) : ex2(from.x - top); };
            const float keep = scale_of(tail);
            value.x *= keep, value.y *= keep, value.z *= keep, value.w *= keep;
            tail = make_float2(top, tail.y * keep);
#pragma unroll
            for (uint32_t i = 0; i < N; ++i) {
                const float scale = scale_of(t[i]);
                value.x = fmaf(scale, v[i].x, value.x), value.y = fmaf(scale, v[i].y, value.y);
                value.z = fmaf(scale, v[i].z, value.z), value.w = fmaf(scale, v[i].w, value.w);
                tail.y = fmaf(scale, t[i].y, tail.y);
            }
        }
    };
    auto put = [&](const Piece &P, uint32_t col, uint32_t d, float4 v, float weight) {
        const uint32_t r = P.row0 + col;
        if (r >= P.rows) return;
        const float by = weight == 0.0f ? 0.0f : 1.0f / weight;
        uint16_t *const to = A.out + (uint64_t)(P.first_row + r / A.group) * A.out_stride + (uint64_t)(P.head * A.group + r % A.group) * DIM + d;
        const uint32_t lo = C.fp16 ? round16x2<true>(v.x * by, v.y * by) : round16x2<false>(v.x * by, v.y * by);
        const uint32_t hi = C.fp16 ? round16x2<true>(v.z * by, v.w * by) : round16x2<false>(v.z * by, v.w * by);
        if (((uintptr_t)to & 7) == 0) *(uint2 *)to = make_uint2(lo, hi);
        else to[0] = (uint16_t)lo, to[1] = (uint16_t)(lo >> 16), to[2] = (uint16_t)hi, to[3] = (uint16_t)(hi >> 16);
    };
    constexpr uint32_t ITEMS = COLS * DIM / 4;
    const Piece *const all_pieces = &s_piece[0][0];
    const bool there = lane < 2 * W && all_pieces[lane].count != 0;
    const uint64_t begin = there ? all_pieces[lane].begin : 0;
    const uint32_t places = __ballot_sync(kFull, there), ahead = places & ((1u << lane) - 1);
    const uint64_t begin_ahead = __shfl_sync(kFull, begin, 31 - __clz(ahead | 1u));
    const uint32_t runs = __ballot_sync(kFull, there && (ahead == 0 || begin_ahead != begin));
    // the unit that began in front of this CTA, and the one that goes on behind it and began here
    const bool open_lane = (runs >> lane & 1) && (begin < cta_from || begin + all_pieces[lane].count > cta_to);
    const uint32_t open_before = __ballot_sync(kFull, open_lane && begin < cta_from), open_behind = __ballot_sync(kFull, open_lane && begin >= cta_from);
    for (uint32_t item = tid; item < __popc(runs) * ITEMS; item += THREADS) {
        uint32_t left = runs;
        for (uint32_t i = item / ITEMS; i; --i) left &= left - 1;
        const uint32_t run = __ffs(left) - 1, col = item % ITEMS / (DIM / 4), d = item % (DIM / 4) * 4;
        const uint32_t later = runs & ~((2u << run) - 1), members = places & ~((1u << run) - 1) & (later ? (1u << (__ffs(later) - 1)) - 1 : kFull);
        // (a run is every warp's first piece, but for its beginning, which may be a last one)
        const float *const begin_at = (run % 2 ? piece_at(run / 2, 1) : first_pieces + run / 2 * Shape::kPiece) + col * ROW, *const rest_at = first_pieces + run / 2 * Shape::kPiece + col * ROW;
        float4 value;
        float2 tail;
        join(std::integral_constant<uint32_t, 4>(), __popc(members), [&](uint32_t i, float4 &v, float2 &t) {
            const float *const from = i ? rest_at + i * Shape::kPiece : begin_at;
            v = *(const float4 *)(from + d), t = *(const float2 *)(from + DIM);
        }, value, tail);
        if ((open_before | open_behind) >> run & 1) {
            float *const piece = A.partials + (2 * (uint64_t)blockIdx.x + (open_before >> run & 1 ? 0 : 1)) * Shape::kPiece + col * ROW;
            __stcg((float4 *)(piece + d), value);
            if (d == 0) __stcg((float2 *)(piece + DIM), tail);
        } else {
            put(all_pieces[run], col, d, value, tail.y);
        }
    }
    if (!(open_before | open_behind)) return;

    // ---- and units of which more than one CTA has: the last one to arrive adds up
    __syncthreads();                                             // (the CTA's pieces are written)
    if (warp < 2) {
        const uint32_t which = warp ? open_behind : open_before;
        bool last = false;
        if (which) {
            const Piece &P = all_pieces[__ffs(which) - 1];
            const uint32_t first_cta = cta_of(P.begin), count = cta_of(P.begin + P.count - 1) - first_cta + 1;
            if (lane == 0) {
                last = arrive_acq_rel(A.tickets + first_cta) == count - 1;
                if (last) A.tickets[first_cta] = 0;
                s_join[warp] = make_uint2(first_cta, last ? count : 0);
            }
        } else if (lane == 0) {
            s_join[warp] = make_uint2(0, 0);
        }
    }
    __syncthreads();
    for (uint32_t item = tid; item < 2 * ITEMS; item += THREADS) {
        const uint32_t k = item / ITEMS, col = item % ITEMS / (DIM / 4), d = item % (DIM / 4) * 4;
        const uint2 J = s_join[k];
        if (J.y == 0) continue;
        // (the unit's first CTA has its piece in the second place, see above)
        const float *const pieces = A.partials + 2 * (uint64_t)J.x * Shape::kPiece + col * ROW;
        float4 value;
        float2 tail;
        join(std::integral_constant<uint32_t, 8>(), J.y, [&](uint32_t i, float4 &v, float2 &t) {
            const float *const from = pieces + (i ? 2 * i : 1) * Shape::kPiece;
            v = __ldcg((const float4 *)(from + d)), t = __ldcg((const float2 *)(from + DIM));
        }, value, tail);
        put(all_pieces[__ffs(k ? open_behind : open_before) - 1], col, d, value, tail.y);
    }
}

template <int DIM, int NT, bool FINE>
static cudaError_t launch_shape(const AttentionArgs &a, uint32_t sms, cudaStream_t stream) {
    using Shape = AttentionShape<DIM, NT>;
    // (the kernel's arrays: barriers and blocks by stage, starts, pieces, late waits, units to join, up to the 128 bytes that the ring is aligned to)
    constexpr uint32_t kArrays = Shape::kWarps * (Shape::kStages * (2 * sizeof(uint64_t) + 2 * sizeof(uint32_t)) + sizeof(uint64_t) + sizeof(uint32_t) +
                                                  sizeof(Sequence) + 2 * sizeof(Piece) + sizeof(uint32_t)) + 2 * sizeof(uint2);
    static_assert(Shape::kSmem + (kArrays + 127) / 128 * 128 <= 232448, "shared memory of a CTA");
    static_assert(Shape::kPiece <= kAttentionPartial, "a piece's place in the workspace");
    static std::atomic<bool> attr_set[64];   // set twice by racing threads at worst: the call is idempotent
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
        const cudaError_t e = cudaFuncSetAttribute(attention_kernel<DIM, NT, FINE>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape::kSmem);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_set[dev].store(true, std::memory_order_release);
    }
    return launch_behind(attention_kernel<DIM, NT, FINE>, dim3(sms < kAttentionCtas ? sms : kAttentionCtas), Shape::kWarps * 32 + 32, Shape::kSmem, stream, a);
}

// One tile of eight rows where a key head has no more than eight, two where it has (and registers hold them).
template <bool FINE>
static cudaError_t launch_dim(const AttentionArgs &a, uint32_t sms, cudaStream_t stream) {
    const bool two = (uint64_t)a.group * ((a.rows + a.c.sequences - 1) / a.c.sequences) > 8;
    switch (a.c.dim) {
        case 64: return two ? launch_shape<64, 2, FINE>(a, sms, stream) : launch_shape<64, 1, FINE>(a, sms, stream);
        case 96: return two ? launch_shape<96, 2, FINE>(a, sms, stream) : launch_shape<96, 1, FINE>(a, sms, stream);
        case 128: return two ? launch_shape<128, 2, FINE>(a, sms, stream) : launch_shape<128, 1, FINE>(a, sms, stream);
        case 192: return launch_shape<192, 1, FINE>(a, sms, stream);
        default: return launch_shape<256, 1, FINE>(a, sms, stream);
    }
}
cudaError_t launch_attention(const AttentionArgs &a, uint32_t sms, cudaStream_t stream) {
    return a.c.fp16 ? launch_dim<true>(a, sms, stream) : launch_dim<false>(a, sms, stream);
}

}  // namespace huffllm
