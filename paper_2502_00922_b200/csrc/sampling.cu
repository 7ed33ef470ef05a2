// The next token of a row of logits, from a given random number.
//
// What stays is a beginning of the order (largest logit first, lower index first among equals), so it is told by its last logit, the cut, and by
// how many of those equal to it stay; which ones these are, and the draw, go by index and need no order.  A cluster of CTAs has a row, which stays
// in shared memory as far as that goes and else in L2.  2048 bins of equal width in the logit (at most 1/64 in the weight's exponent) count the
// tokens above every edge, and the weights' mass, in whole numbers and so in any order.  The bin in which top_k or top_p end goes to a
// list of the first CTA, which finds the cut by halving the range of its values.  Where top_k is small, the largest logits of parts of the row bound the
// cut from below, and only what is above that bound, a list too, is looked at again.  min_p is a logit, and raises the cut.
//
// Few rows are bound by the way from phase to phase (ten barriers of the cluster): 32000 logits 17.8 us.  Many are bound by instructions, 20 a
// logit where top_k bounds the cut, else 80: 200 rows of 150001 in BF16 54 us, 64 of 128000 in fp32, top_p alone, 48 us (read once: 9 and 5 us).
// Weights are fp32: of 25600 rows of 128000 tokens five fell to the other side of a border than 64 bits (two with weights in 64, 65 us for 64 of them).
// Four CTAs an SM of 256 threads, as the phases of one wait for each other: 64 x 128000 with two of 512 threads and the row in shared memory 67 us.
#include <cooperative_groups.h>
#include <cuda_runtime.h>

#include "decode_common.cuh"
#include "decode_step.h"
#include "epilogue.cuh"

namespace cg = cooperative_groups;

namespace huffllm {

constexpr uint32_t kSampleThreads = 256, kSampleEach = 4,   // CTAs an SM has room for
                    kSampleWarps = kSampleThreads / 32;
constexpr uint32_t kBins = 2048;
constexpr uint32_t kBeyond = kBins + 1;                // (in the place of a bin's number) what lies beyond all of them
constexpr uint32_t kMostList = 2 * kBins;              // a bin with fewer logits is searched in shared memory, in a list that lies where the bins were
constexpr uint32_t kShortList = 256, kMostNear = 2048;
constexpr uint32_t kMostCluster = 8;
constexpr uint32_t kFull = 0xFFFFFFFFu;

// Ascending with the value, both zeros alike.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x == 0.0f ? 0.0f : x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key); }

// Values of a 16-byte piece, widened
template <int TYPE>
struct Piece16 {
    static constexpr int N = TYPE == 0 ? 4 : 8;
    float x[N];
    __device__ __forceinline__ explicit Piece16(uint4 v) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (TYPE == 0) x[i] = __uint_as_float(w[i]);
            else x[2 * i] = widen16<TYPE == 2>((uint16_t)w[i]), x[2 * i + 1] = widen16<TYPE == 2>((uint16_t)(w[i] >> 16));
        }
    }
};

// The largest and the smallest value of a piece (a NaN is none).
template <int TYPE>
__device__ __forceinline__ float piece_max(uint4 v) {
    if constexpr (TYPE == 0) return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
    using Two = std::conditional_t<TYPE == 1, __nv_bfloat162, __half2>;
    const Two m = __hmax2(__hmax2(*(const Two *)&v.x, *(const Two *)&v.y), __hmax2(*(const Two *)&v.z, *(const Two *)&v.w));
    return fmaxf(widen16<TYPE == 2>((uint16_t)*(const uint32_t *)&m), widen16<TYPE == 2>((uint16_t)(*(const uint32_t *)&m >> 16)));
}
template <int TYPE>
__device__ __forceinline__ float piece_min(uint4 v) {
    if constexpr (TYPE == 0) return fminf(fminf(__uint_as_float(v.x), __uint_as_float(v.y)), fminf(__uint_as_float(v.z), __uint_as_float(v.w)));
    using Two = std::conditional_t<TYPE == 1, __nv_bfloat162, __half2>;
    const Two m = __hmin2(__hmin2(*(const Two *)&v.x, *(const Two *)&v.y), __hmin2(*(const Two *)&v.z, *(const Two *)&v.w));
    return fminf(widen16<TYPE == 2>((uint16_t)*(const uint32_t *)&m), widen16<TYPE == 2>((uint16_t)(*(const uint32_t *)&m >> 16)));
}

// Which values of a piece are `floor` or more, which is a value of the type: bits 0 .. 3, or of 16-bit values i and i + 16 for the lower and
// upper half of word i; and the value that such a bit stands for.
template <int TYPE>
__device__ __forceinline__ uint32_t at_least(uint4 v, float floor) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t hits = 0;
    if constexpr (TYPE == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) hits |= __uint_as_float(w[i]) >= floor ? 1u << i : 0u;
    } else {
        using Two = std::conditional_t<TYPE == 1, __nv_bfloat162, __half2>;
        const uint32_t both = round16<TYPE == 2>(floor) * 0x10001u;
#pragma unroll
        for (int i = 0; i < 4; ++i) hits |= __hge2_mask(*(const Two *)&w[i], *(const Two *)&both) & 0x10001u << i;
    }
    return hits;
}
template <int TYPE>
__device__ __forceinline__ float value_at(uint4 v, uint32_t bit) {
    const uint32_t lo = bit & 1 ? v.y : v.x, hi = bit & 1 ? v.w : v.z, w = bit & 2 ? hi : lo;
    if constexpr (TYPE == 0) return __uint_as_float(w);
    return widen16<TYPE == 2>((uint16_t)(bit & 16 ? w >> 16 : w));
}

struct alignas(16) SampleShared {
    uint32_t count[kBins];                             // a CTA's bins; later, in the first CTA, the list
    uint32_t below[kBins];
    uint32_t all_count[kBins];                         // the first CTA: all CTAs' bins
    float all_mass[kBins];
    union {
        struct {
            float near[kMostNear];                     // a CTA's logits that may be above the cut, where top_k is small,
            uint32_t near_piece[kMostNear];            // and the pieces that have them
        };
        uint64_t below_wide[kBins];                    // or `below` of a CTA with so many logits that 32 bits would not hold it
    };
    double warp_mass[kSampleWarps], scan_mass[kSampleWarps];
    uint32_t warp_equal[kSampleWarps], scan_count[kSampleWarps], sums[2][kSampleWarps];
    float warp_top[kSampleWarps], warp_least[kSampleWarps];
    float cta_top, cta_least;
    double table_mass[kMostCluster * kSampleWarps];
    uint32_t table_equal[kMostCluster * kSampleWarps];
    uint32_t found_bin, found_count, listed[2], nears, wide;
    double found_mass, min_reach;
    struct {
        uint32_t bin, lowest;
        double want;
    } named[2];                                        // what the first CTA searches: by count, by mass
    uint32_t draw_stretch, draw_equal;                 // where the draw ends; of the equals in front of it, the mass there, and what it has to exceed
    double draw_from, draw_aim;
    float cut;                                         // the outcome: logits above it stay, and `ties` of those that equal it
    uint32_t ties;
};

// One row, as a CTA sees it: `pieces` pieces of 16 bytes, of which the first `kept` lie in shared memory.  Values outside the CTA's part of the
// row are NaN, which is neither above nor equal to anything.
template <int TYPE>
struct RowPart {
    static constexpr int N = Piece16<TYPE>::N;
    using Raw = std::conditional_t<TYPE == 0, uint32_t, uint16_t>;
    const Raw *first;                                  // the CTA's first value in memory
    uint4 *data;
    uint32_t count, phase, pieces, kept;
    __device__ __forceinline__ uint4 from_memory(uint32_t piece) const {
        const int64_t at = (int64_t)piece * N - phase;
        if (at >= 0 && at + N <= count) return __ldcg((const uint4 *)(first + at));
        Raw v[N];
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = at + j >= 0 && at + j < count ? __ldcg(first + at + j) : (Raw)0x7FFFFFFFu;
        uint4 r;
        if constexpr (TYPE == 0) r = make_uint4(v[0], v[1], v[2], v[3]);
        else r = make_uint4(v[0] | (uint32_t)v[1] << 16, v[2] | (uint32_t)v[3] << 16, v[4] | (uint32_t)v[5] << 16, v[6] | (uint32_t)v[7] << 16);
        return r;
    }
    __device__ __forceinline__ uint4 raw(uint32_t i) const { return i < kept ? data[i] : from_memory(i); }
    // f(piece, its number) for the pieces first, first + step .. below end; four are on their way together (they may come from L2), and behind
    // every four g().
    template <typename F, typename G>
    __device__ __forceinline__ void each(uint32_t first, uint32_t end, uint32_t step, F f, G g) const {
        for (uint32_t i0 = first; i0 < end; i0 += 4 * step) {
            uint4 v[4];
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) v[j] = i0 + j * step < end ? raw(i0 + j * step) : make_uint4(kFull, kFull, kFull, kFull);
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) f(v[j], i0 + j * step);
            g();
        }
    }
    template <typename F>
    __device__ __forceinline__ void each(uint32_t first, uint32_t end, uint32_t step, F f) const {
        each(first, end, step, f, [] {});
    }
};

__device__ __forceinline__ float exp2_approx(float x) {   // off by 2^-22 of itself
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float warp_max(float v) {
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kFull, v, o));
    return v;
}
__device__ __forceinline__ float warp_min(float v) {
    for (int o = 16; o; o >>= 1) v = fminf(v, __shfl_xor_sync(kFull, v, o));
    return v;
}

template <int TYPE>
__global__ void __launch_bounds__(kSampleThreads, kSampleEach) sample_kernel(const __grid_constant__ SamplingArgs A) {
    extern __shared__ __align__(16) uint8_t dynamic[];
    SampleShared &S = *(SampleShared *)dynamic;
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t tid = threadIdx.x, lane = tid % 32, warp = tid / 32, ctas = cluster.num_blocks(), rank = cluster.block_rank();
    const uint32_t row = blockIdx.x / ctas;
    SampleShared &S0 = *cluster.map_shared_rank(&S, 0);
    pdl_launch_dependents();
    for (uint32_t i = tid; i < kBins; i += kSampleThreads) S.count[i] = S.below[i] = 0;
    pdl_wait_prior_grid();

    RowPart<TYPE> R;
    using Raw = typename RowPart<TYPE>::Raw;
    const uint32_t i0 = min(A.vocab, rank * A.part);
    R.first = (const Raw *)A.logits + row * A.stride + i0;
    R.data = (uint4 *)(dynamic + sizeof(SampleShared));
    R.count = min(A.vocab - i0, A.part);
    R.phase = (uint32_t)((uintptr_t)R.first % 16 / sizeof(Raw));
    R.pieces = R.count ? (R.phase + R.count + R.N - 1) / R.N : 0;
    R.kept = min(R.pieces, A.kept_pieces);

    const float t_given = A.temperature ? __ldcg(A.temperature + row) : 1.0f, p = A.top_p ? __ldcg(A.top_p + row) : 1.0f, u = __ldcg(A.uniform + row);
    const float min_p = A.min_p ? __ldcg(A.min_p + row) : 0.0f;
    const int32_t k_given = A.top_k ? __ldcg(A.top_k + row) : 0;
    // A weight beyond the bins is below exp(-32) < 2^-46.  Those of a whole row are less than any draw but one next to 0 or to 1 leaves on either side.
    const float beyond = (float)A.vocab * 0x1p-46f;
    const bool at_ends = !(u > beyond && u < 1.0f - beyond);
    const bool first_only = !(t_given > 0.0f) || p <= 0.0f || k_given == 1;
    const float temperature = first_only ? 1.0f : fminf(fmaxf(t_given, 1e-30f), 1e30f);       // (beyond, its products leave fp32)

    // ---- the row into shared memory; its largest and smallest logit
    float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, least = INFINITY;   // of four parts of the thread's logits
    for (uint32_t i0 = tid; i0 < R.pieces; i0 += 4 * kSampleThreads) {
        uint4 v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t i = i0 + j * kSampleThreads;
            v[j] = i < R.pieces ? R.from_memory(i) : make_uint4(kFull, kFull, kFull, kFull);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t i = i0 + j * kSampleThreads;
            if (i < R.kept) R.data[i] = v[j];
            tops[j] = fmaxf(tops[j], piece_max<TYPE>(v[j]));
            least = fminf(least, piece_min<TYPE>(v[j]));
        }
    }
    float top = warp_max(fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])));
    least = warp_min(least);
    if (lane == 0) S.warp_top[warp] = top, S.warp_least[warp] = least;
    __syncthreads();
    if (warp == 0) {
        top = warp_max(lane < kSampleWarps ? S.warp_top[lane] : -INFINITY);
        least = warp_min(lane < kSampleWarps ? S.warp_least[lane] : INFINITY);
        // min_p as a distance between logits, in 64 bits (a weight in 32 is 1 for what lies next to the largest)
        if (lane == 0 && min_p > 0.0f) S.min_reach = min_p < 1.0f ? (double)temperature * log((double)min_p) : 0.0;
        if (lane == 0) S.cta_top = top, S.cta_least = least, S.listed[0] = S.listed[1] = S.nears = S.wide = 0;
    }
    cluster.sync();
    {
        const SampleShared &other = *cluster.map_shared_rank(&S, lane % ctas);
        top = warp_max(other.cta_top);
        least = warp_min(other.cta_least);
    }
    if (top == -INFINITY) {                            // (every CTA of the row comes here)
        if (rank == 0 && tid == 0) A.tokens[row] = -1;
        cluster.sync();
        return;
    }
    // Exponents of weights in bins: most 1/64 wide, narrower where the row's logits are closer together (and none is minus infinity).
    const float scale = fmaxf(64.0f / temperature, fminf((float)(kBins - 1) / (top - least), 1e30f));
    const float width = 1.0f / (scale * temperature), to_log2 = -1.4426950408889634f / temperature;
    auto place = [&](float x) { return (top - x) * scale; };
    // (of the largest, were it infinite, this is no number: what equals the cut takes the cut's)
    auto weight = [&](float x) { return exp2_approx((top - x) * to_log2); };
    // The bin of a place below kBins (2^23 and more has no fraction, and its low bits are the whole number; conversions go through a slower
    // pipe), and a weight's distance from that of the bin's upper edge, in 2^-22 of it: 1 - exp(-r) for r up to 1/64.
    auto bin_of = [](float place) { return __float_as_uint(__fadd_rd(place, 8388608.0f)) & (2 * kBins - 1); };
    auto below_edge = [&](float place) {
        const float r = (place - (__fadd_rd(place, 8388608.0f) - 8388608.0f)) * width;
        return __float_as_uint(fmaf(r * (1.0f - r * (0.5f - r * 0.16666667f)), 4194304.0f, 12582912.0f)) & 0x1FFFFu;
    };

    float cut = -INFINITY;                             // (what equals minus infinity has no weight)
    uint32_t ties = 0;
    bool by_near = false;                              // what stays is in the list of near logits
    const bool by_count = !first_only && k_given > 0 && (uint32_t)k_given < A.vocab, by_mass = !first_only && p < 1.0f;
    const bool infinite = top == INFINITY;             // (equal weights: how many stay shows when all of them are counted, for the draw)
    if (first_only || infinite) {
        cut = top;
        ties = 1;
    } else if (by_count || by_mass) {
        // ---- the bins
        const bool two_sums = by_count || A.part >= 16384, may_be_wide = by_mass && A.part > 65536;
        const float units = __uint_as_float((127u + min(22u, (uint32_t)__clz(A.part))) << 23);
        // Where top_k is small, most of the row need not be looked at closely: of the largest logits of the threads' parts, which are that many
        // tokens, the top_k-th largest is not above the cut.  (Halving a range ten times is near enough.  200 x 150001 in BF16, top_k 400: 134 -> 55 us.)
        float floor = -INFINITY;
        if (by_count && (uint32_t)k_given <= kSampleThreads * 3 && (uint32_t)k_given < R.count / 8) {
            float high = top;                          // `floor` or more have so many parts or more
            for (uint32_t turn = 0; turn < 11; ++turn) {
                const float mid = turn == 0 ? top - 16.0f * temperature : 0.5f * (floor + high);
                const uint32_t count = __reduce_add_sync(kFull, (tops[0] >= mid) + (tops[1] >= mid) + (tops[2] >= mid) + (tops[3] >= mid));
                if (lane == 0) S.sums[turn & 1][warp] = count;
                __syncthreads();
                if (__reduce_add_sync(kFull, lane < kSampleWarps ? S.sums[turn & 1][lane] : 0u) >= (uint32_t)k_given) floor = mid;
                else high = mid;
                if (floor == -INFINITY) break;
            }
            if constexpr (TYPE == 1) floor = __bfloat162float(__float2bfloat16_rd(floor));
            if constexpr (TYPE == 2) floor = __half2float(__float2half_rd(floor));
            __syncthreads();
        }
        const uint32_t counts_at = (uint32_t)__cvta_generic_to_shared(S.count), below_at = (uint32_t)__cvta_generic_to_shared(S.below);
        // (with predicates: a branch for every logit costs more than what is behind it)
        auto count_one = [&](float x) {
            const float at = place(x);
            const uint32_t bin = bin_of(at) * 4;
            asm volatile("{\n\t.reg .pred p;\n\tsetp.lt.f32 p, %0, %1;\n\t@p red.shared.add.u32 [%2], 1;\n\t}" ::"f"(at), "f"((float)kBins), "r"(counts_at + bin)
                         : "memory");
            if (by_mass)
                asm volatile("{\n\t.reg .pred p;\n\tsetp.lt.f32 p, %0, %1;\n\t@p red.shared.add.u32 [%2], %3;\n\t}" ::"f"(at), "f"((float)kBins), "r"(below_at + bin),
                             "r"(below_edge(at))
                             : "memory");
        };
        // Mass alone, in one addition: a weight in `units` of its bin's upper edge, as many as the CTA's logits leave of 32 bits (2^18 or more where a CTA
        // has less than 16384 logits: a weight is off by 2^-19 of itself at most).  units exp(-r) is a polynomial in how far the place is in its bin.
        const float c1 = -units * width, c2 = 0.5f * units * width * width, c3 = -units * width * width * width / 6.0f;
        auto weigh_one = [&](float x) {
            const float at = place(x), whole = __fadd_rd(at, 8388608.0f), f = at - (whole - 8388608.0f);
            const uint32_t bin = (__float_as_uint(whole) & (2 * kBins - 1)) * 4;
            const uint32_t w = __float_as_uint(fmaf(fmaf(fmaf(c3, f, c2), f, c1), f, units + 8388608.0f)) & 0x7FFFFFu;
            asm volatile("{\n\t.reg .pred p;\n\tsetp.lt.f32 p, %0, %1;\n\t@p red.shared.add.u32 [%2], %3;\n\t}" ::"f"(at), "f"((float)kBins), "r"(below_at + bin), "r"(w)
                         : "memory");
        };
        if (floor > -INFINITY) {
            R.each(tid, R.pieces, kSampleThreads, [&](uint4 v, uint32_t i) {
                uint32_t hits = at_least<TYPE>(v, floor);
                if (!hits) return;
                uint32_t to = atomicAdd(&S.nears, __popc(hits));
                for (; hits; hits &= hits - 1, ++to)
                    if (to < kMostNear) S.near[to] = value_at<TYPE>(v, __ffs(hits) - 1), S.near_piece[to] = i;
            });
            __syncthreads();
        }
        const uint32_t nears = S.nears;
        by_near = floor > -INFINITY && nears <= kMostNear;
        if (by_near) {
            for (uint32_t i = tid; i < nears; i += kSampleThreads) count_one(S.near[i]);
        } else {
            // (distances are below 2^16: 2^16 logits add up within 32 bits; behind so many, the sums go to 64)
            const bool wide = may_be_wide && R.count > 65536;
            const uint32_t chunk = wide ? 65536 / R.N : R.pieces;
            for (uint32_t from = 0; from < R.pieces; from += chunk) {
                R.each(from + tid, min(R.pieces, from + chunk), kSampleThreads, [&](uint4 v, uint32_t) {
                    const Piece16<TYPE> x(v);
#pragma unroll
                    for (int e = 0; e < R.N; ++e) {
                        if (two_sums) count_one(x.x[e]);
                        else weigh_one(x.x[e]);
                    }
                });
                if (!wide) break;
                __syncthreads();
                for (uint32_t i = tid; i < kBins; i += kSampleThreads) S.below_wide[i] = (from ? S.below_wide[i] : 0) + S.below[i], S.below[i] = 0;
                __syncthreads();
            }
            if (wide && tid == 0) S.wide = 1;
        }
        cluster.sync();
        const uint32_t share = kBins / ctas;
        for (uint32_t i = tid; i < share; i += kSampleThreads) {
            const uint32_t bin = rank * share + i;
            uint32_t count = 0;
            uint64_t below = 0;
            for (uint32_t r = 0; r < ctas; ++r) {
                const SampleShared &other = *cluster.map_shared_rank(&S, r);
                count += other.count[bin];
                below += may_be_wide && other.wide ? other.below_wide[bin] : other.below[bin];
            }
            S0.all_count[bin] = count;
            S0.all_mass[bin] = expf(-(float)bin * width) * (float)(two_sums ? (double)count - (double)below * 0x1p-22 : (double)below / units);
        }
        cluster.sync();

        // ---- the first CTA: up to where in the bins
        constexpr uint32_t PER = kBins / kSampleThreads;
        uint32_t count_to = 0, counts[PER] = {};
        double mass_to = 0.0;
        float masses[PER] = {};
        if (rank == 0) {
            uint32_t c = 0;
            double m = 0.0;
#pragma unroll
            for (uint32_t j = 0; j < PER; ++j) {
                counts[j] = S.all_count[tid * PER + j];
                masses[j] = S.all_mass[tid * PER + j];
                c += counts[j];
                m += masses[j];
            }
            uint32_t ci = c;
            double mi = m;
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t cu = __shfl_up_sync(kFull, ci, o);
                const double mu = __shfl_up_sync(kFull, mi, o);
                if (lane >= o) ci += cu, mi += mu;
            }
            if (lane == 31) S.scan_count[warp] = ci, S.scan_mass[warp] = mi;
            __syncthreads();
            count_to = ci - c;
            mass_to = mi - m;
            for (uint32_t w = 0; w < warp; ++w) count_to += S.scan_count[w], mass_to += S.scan_mass[w];
        }
        // The bin in which the count, or the mass, reaches what is wanted (kBins: in none); `limit`: bins from there on do not count.
        auto find = [&](bool counted, uint32_t want_count, double want_mass, uint32_t limit) {
            if (tid == 0) S.found_bin = kBins;
            __syncthreads();
            uint32_t c = count_to;
            double m = mass_to;
#pragma unroll
            for (uint32_t j = 0; j < PER; ++j) {
                const uint32_t c1 = c + counts[j], bin = tid * PER + j;
                const double m1 = m + masses[j];
                if (bin < limit && (counted ? c < want_count && c1 >= want_count : m < want_mass && m1 >= want_mass))
                    S.found_bin = bin, S.found_count = c, S.found_mass = m;
                c = c1;
                m = m1;
            }
            __syncthreads();
        };
        float *const list = (float *)S.count;
        auto lies_in = [&](float x, uint32_t bin) {
            const float at = place(x);
            return bin == kBeyond ? at >= (float)kBins : at < (float)kBins && bin_of(at) == bin;
        };
        // All of a bin's logits into the first CTA's list.
        auto gather = [&](uint32_t bin, uint32_t which) {
            float *const list0 = (float *)S0.count;
            auto in_bin = [&](float x) { return lies_in(x, bin); };
            if (by_near) {                             // (beyond the bins: of no CTA, as its near logits alone are top_k)
                for (uint32_t i = tid; i < nears; i += kSampleThreads) {
                    if (!in_bin(S.near[i])) continue;
                    const uint32_t to = atomicAdd(&S0.listed[which], 1u);
                    if (to < kMostList) list0[to] = S.near[i];
                }
                return;
            }
            // (most pieces have none within half a bin of its middle, give or take what rounding moves its edges)
            const float middle = top - ((float)bin + 0.5f) / scale, reach = 0.505f / scale + (fabsf(middle) + fabsf(top)) * 1e-6f;
            R.each(tid, R.pieces, kSampleThreads, [&](uint4 v, uint32_t) {
                const Piece16<TYPE> x(v);
                float nearest = INFINITY;
#pragma unroll
                for (int e = 0; e < R.N; ++e) nearest = fminf(nearest, fabsf(x.x[e] - middle));
                if (nearest > reach && bin != kBeyond) return;
                uint32_t hits = 0;
#pragma unroll
                for (int e = 0; e < R.N; ++e) hits |= in_bin(x.x[e]) ? 1u << e : 0u;
                if (hits) {
                    uint32_t to = atomicAdd(&S0.listed[which], __popc(hits));
#pragma unroll
                    for (int e = 0; e < R.N; ++e)
                        if (hits >> e & 1) {
                            if (to < kMostList) list0[to] = x.x[e];
                            ++to;
                        }
                }
            });
        };
        // Searches the keys of a bin: the first key, from above, at which the count (or the mass, in 2^-20 of the bin's upper edge) of all
        // keys down to it reaches `want`.  above: of the keys above it; equal: how many have it.
        struct Edge {
            uint32_t key, equal;
            double above;
            bool by_row;                               // every CTA has found it
        };
        auto mass20 = [&](float x) { return 1048576u - (below_edge(place(x)) >> 2); };
        auto block_sum = [&](uint32_t v, uint32_t turn) {
            v = __reduce_add_sync(kFull, v);
            if (lane == 0) S.sums[turn & 1][warp] = v;
            __syncthreads();
            return __reduce_add_sync(kFull, lane < kSampleWarps ? S.sums[turn & 1][lane] : 0u);
        };
        // (a short list: every warp by itself)
        auto search_short = [&](uint32_t n, bool counted, double want, uint32_t lowest) -> Edge {
            constexpr uint32_t EACH = kShortList / 32;
            const uint32_t whole_want = (uint32_t)fmin(ceil(want), 4294967295.0);
            uint32_t key[EACH], part[EACH], low = kFull, high = 0;
#pragma unroll
            for (uint32_t j = 0; j < EACH; ++j) {
                const uint32_t i = lane + j * 32;
                key[j] = 0, part[j] = 0;
                if (i < n) {
                    key[j] = key_of(list[i]);
                    part[j] = counted ? 1u : mass20(list[i]);
                    low = min(low, key[j]);
                    high = max(high, key[j]);
                }
            }
            low = max(__reduce_min_sync(kFull, low), lowest) - 1;
            high = __reduce_max_sync(kFull, high);
            auto above = [&](uint32_t mid) {
                uint32_t v = 0;
#pragma unroll
                for (uint32_t j = 0; j < EACH; ++j) v += key[j] > mid ? part[j] : 0u;
                return __reduce_add_sync(kFull, v);
            };
            while (high - low > 1) {
                const uint32_t mid = low + (high - low) / 2;
                if (above(mid) < whole_want) high = mid;
                else low = mid;
            }
            uint32_t v = 0;
#pragma unroll
            for (uint32_t j = 0; j < EACH; ++j) v += key[j] == high;
            return Edge{high, __reduce_add_sync(kFull, v), (double)above(high), false};
        };
        auto search_list = [&](uint32_t n, bool counted, double want, uint32_t lowest) -> Edge {
            if (n <= kShortList) return search_short(n, counted, want, lowest);
            constexpr uint32_t EACH = kMostList / kSampleThreads;
            const uint32_t whole_want = (uint32_t)fmin(ceil(want), 4294967295.0);
            uint32_t key[EACH], part[EACH], low = kFull, high = 0;
#pragma unroll
            for (uint32_t j = 0; j < EACH; ++j) {
                const uint32_t i = tid + j * kSampleThreads;
                key[j] = 0, part[j] = 0;
                if (i < n) {
                    key[j] = key_of(list[i]);
                    part[j] = counted ? 1u : mass20(list[i]);
                    low = min(low, key[j]);
                    high = max(high, key[j]);
                }
            }
            low = __reduce_min_sync(kFull, low);
            high = __reduce_max_sync(kFull, high);
            if (lane == 0) S.sums[0][warp] = low, S.sums[1][warp] = high;
            __syncthreads();
            low = __reduce_min_sync(kFull, lane < kSampleWarps ? S.sums[0][lane] : kFull);
            high = __reduce_max_sync(kFull, lane < kSampleWarps ? S.sums[1][lane] : 0u);
            __syncthreads();
            low = max(low, lowest) - 1;                // `want` or more above it (or as much as there is); less above `high`
            uint32_t turn = 0;
            auto above = [&](uint32_t mid) {
                uint32_t v = 0;
#pragma unroll
                for (uint32_t j = 0; j < EACH; ++j) v += key[j] > mid ? part[j] : 0u;
                return block_sum(v, turn++);
            };
            while (high - low > 1) {
                const uint32_t mid = low + (high - low) / 2;
                if (above(mid) < whole_want) high = mid;
                else low = mid;
            }
            Edge e;
            e.key = high;
            e.above = (double)above(high);
            uint32_t v = 0;
#pragma unroll
            for (uint32_t j = 0; j < EACH; ++j) v += key[j] == high;
            e.equal = block_sum(v, turn++);
            e.by_row = false;
            __syncthreads();
            return e;
        };
        // The same where a bin has more logits than the list: every CTA goes through its part of the row at every turn.
        enum { kCountAbove, kMassAbove, kCountEqual };
        auto row_total = [&](uint32_t bin, uint32_t edge, int what) -> double {
            uint64_t v = 0;
            R.each(tid, R.pieces, kSampleThreads, [&](uint4 piece, uint32_t) {
                const Piece16<TYPE> x(piece);
#pragma unroll
                for (int e = 0; e < R.N; ++e) {
                    if (!lies_in(x.x[e], bin)) continue;
                    const uint32_t key = key_of(x.x[e]);
                    if (what == kCountEqual ? key == edge : key > edge) v += what == kMassAbove ? mass20(x.x[e]) : 1u;
                }
            });
            for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(kFull, v, o);
            if (lane == 0) S.warp_mass[warp] = (double)v;
            cluster.sync();
            double sum = 0.0;
            for (uint32_t r = 0; r < ctas; ++r) {
                const SampleShared &other = *cluster.map_shared_rank(&S, r);
                for (uint32_t w = 0; w < kSampleWarps; ++w) sum += other.warp_mass[w];
            }
            cluster.sync();
            return sum;
        };
        auto search_row = [&](uint32_t bin, bool counted, double want, uint32_t lowest) -> Edge {
            uint32_t low = max(key_of(-INFINITY), lowest) - 1, high = key_of(top);
            while (high - low > 1) {
                const uint32_t mid = low + (high - low) / 2;
                if (row_total(bin, mid, counted ? kCountAbove : kMassAbove) < want) high = mid;
                else low = mid;
            }
            Edge e;
            e.key = high;
            e.above = row_total(bin, high, counted ? kCountAbove : kMassAbove);
            e.equal = (uint32_t)row_total(bin, high, kCountEqual);
            e.by_row = true;
            return e;
        };
        // Gathers and searches a bin that the first CTA names (kBins: none).
        uint32_t gathered = kBins, list_of = 0;
        auto search = [&](uint32_t bin0, bool counted, double want0, uint32_t lowest0) -> Edge {
            if (rank == 0 && tid < ctas) {
                auto &to = cluster.map_shared_rank(&S, tid)->named[counted ? 0 : 1];
                to.bin = bin0, to.want = want0, to.lowest = lowest0;
            }
            cluster.sync();
            const auto &named = S.named[counted ? 0 : 1];
            const uint32_t bin = named.bin, lowest = named.lowest;
            const double want = named.want;
            Edge e{0, 0, 0.0, false};
            if (bin == kBins) return e;
            if (bin != gathered) {
                list_of = counted ? 0 : 1;
                gather(bin, list_of);
                cluster.sync();
                gathered = bin;
            }
            const uint32_t n = S0.listed[list_of];
            if (n >= kMostList) return search_row(bin, counted, want, lowest);
            if (rank == 0) e = search_list(n, counted, want, lowest);
            return e;
        };

        double mass = 0.0;                             // of what top_k leaves
        uint32_t limit = kBins, lowest = 0;
        bool unfilled = false;
        if (rank == 0)
            for (uint32_t w = 0; w < kSampleWarps; ++w) mass += S.scan_mass[w];
        if (by_count) {
            uint32_t bin = kBins, before = 0;
            double mass_before = 0.0;
            if (rank == 0) {
                find(true, (uint32_t)k_given, 0.0, kBins);
                bin = S.found_bin, before = S.found_count, mass_before = S.found_mass;
                __syncthreads();
                // Fewer than top_k in the bins.  Which of the others stay shows in a draw at one of the ends alone (and not where top_p cuts, which is within
                // the bins): else the cut is the bins' far end, found without a look at the row.
                if (bin == kBins && at_ends && !by_mass) {
                    bin = kBeyond, before = 0;
                    for (uint32_t w = 0; w < kSampleWarps; ++w) before += S.scan_count[w];
                }
                unfilled = bin == kBins;
            }
            const Edge e = search(bin, true, (double)((uint32_t)k_given - before), 0);
            const double row_mass = e.by_row && by_mass ? row_total(S.named[0].bin, e.key, kMassAbove) : 0.0;
            if (rank == 0 && bin != kBins) {
                cut = value_of(e.key);
                ties = (uint32_t)k_given - before - (uint32_t)e.above;
            }
            if (rank == 0 && bin < kBins) {
                limit = bin + 1;
                lowest = e.key;
                if (by_mass) {
                    // the mass of what stays of the bin: its keys above the cut, and the ties
                    double inside = row_mass;
                    if (!e.by_row) {
                        uint32_t v = 0;
                        for (uint32_t i = tid; i < S.listed[0]; i += kSampleThreads) v += key_of(list[i]) > e.key ? mass20(list[i]) : 0u;
                        inside = (double)block_sum(v, 0);
                        __syncthreads();
                    }
                    mass = mass_before + exp((double)(-(float)bin * width)) * 0x1p-20 * (inside + (double)ties * mass20(cut));
                }
            }
        }
        if (by_mass) {
            uint32_t bin = kBins;
            double want = (double)p * mass, part = 0.0;
            if (rank == 0) {
                find(false, 0, want, limit);
                bin = S.found_bin;
                part = (want - S.found_mass) * exp((double)((float)bin * width)) * 0x1p20;
                __syncthreads();
            }
            const Edge e = search(bin, false, part, bin + 1 == limit ? lowest : 0);
            if (rank == 0 && bin < kBins) {
                const uint32_t have = bin + 1 == limit && e.key == lowest ? ties : e.equal;
                const float edge = value_of(e.key);
                const double need = ceil((part - e.above) / (double)mass20(edge));
                cut = edge;
                ties = (uint32_t)fmin(fmax(need, 1.0), (double)have);
            }
        }
        if (unfilled && cut == -INFINITY) {
            uint32_t low = key_of(-INFINITY), high = key_of(top);          // the largest value whose place is beyond the bins
            while (high - low > 1) {
                const uint32_t mid = low + (high - low) / 2;
                if (place(value_of(mid)) < (float)kBins) high = mid;
                else low = mid;
            }
            cut = value_of(low);
        }
        __syncthreads();
        if (rank == 0 && tid < ctas) {
            SampleShared &other = *cluster.map_shared_rank(&S, tid);
            other.cut = cut, other.ties = ties;
        }
        cluster.sync();
        cut = S.cut;
        ties = S.ties;
    }

    if (min_p > 0.0f) {
        const float least = __double2float_ru((double)top + S.min_reach);
        if (least > cut) cut = nextafterf(least, -INFINITY), ties = 0;
    }

    // ---- the draw, in the order of indexes: warps have stretches of the row, lanes pieces of 16 bytes that follow each other
    // a warp's mass above the cut of a stretch, and how many equal it, into the warp's place
    auto sum_stretch = [&](uint32_t from, uint32_t to) {
        float sum = 0.0f;                              // of four pieces; a lane may have so many that 32 bits do not do
        double m = 0.0;
        uint32_t equal = 0;
        R.each(from + lane, to, 32, [&](uint4 v, uint32_t) {
            if (!(piece_max<TYPE>(v) >= cut)) return;
            const Piece16<TYPE> x(v);
#pragma unroll
            for (int e = 0; e < R.N; ++e) {
                const float w = weight(x.x[e]);        // (a select costs less than a branch)
                sum += x.x[e] > cut ? w : 0.0f;
                equal += x.x[e] == cut;
            }
        }, [&] { m += sum, sum = 0.0f; });
        for (int o = 16; o; o >>= 1) m += __shfl_xor_sync(kFull, m, o);
        equal = __reduce_add_sync(kFull, equal);
        if (lane == 0) S.warp_mass[warp] = m, S.warp_equal[warp] = equal;
    };
    const uint32_t stretch = (R.pieces + kSampleWarps * 32 - 1) / (kSampleWarps * 32) * 32;
    if (by_near) {
        // (the list is in no order: masses in whole numbers, 2^-40)
        uint64_t sum = 0;
        uint32_t equal = 0;
        for (uint32_t i = lane; i < S.nears; i += 32) {
            if (S.near_piece[i] / stretch != warp) continue;
            const float x = S.near[i];
            if (x > cut) sum += (uint64_t)((double)weight(x) * 0x1p40);
            equal += x == cut;
        }
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(kFull, sum, o);
        equal = __reduce_add_sync(kFull, equal);
        if (lane == 0) S.warp_mass[warp] = (double)sum * 0x1p-40, S.warp_equal[warp] = equal;
    } else {
        sum_stretch(min(R.pieces, warp * stretch), min(R.pieces, (warp + 1) * stretch));
    }
    cluster.sync();
    for (uint32_t i = tid; i < ctas * kSampleWarps; i += kSampleThreads) {
        const SampleShared &other = *cluster.map_shared_rank(&S, i / kSampleWarps);
        S.table_mass[i] = other.warp_mass[i % kSampleWarps];
        S.table_equal[i] = other.warp_equal[i % kSampleWarps];
    }
    cluster.sync();                                    // (the last look at another CTA's shared memory)
    const float cut_weight = cut == -INFINITY ? 0.0f : cut == top ? 1.0f : weight(cut);
    // the first warp: the stretch in which the mass exceeds what is drawn; a lane has some that follow each other
    constexpr uint32_t STRETCHES = kMostCluster * kSampleWarps / 32;    // of a lane
    if (warp == 0) {
        const uint32_t stretches = ctas * kSampleWarps;
        uint32_t eq[STRETCHES], eq_to = 0;
        double m[STRETCHES], m_to = 0.0;
#pragma unroll
        for (uint32_t j = 0; j < STRETCHES; ++j) {
            const uint32_t i = lane * STRETCHES + j;
            eq[j] = i < stretches ? S.table_equal[i] : 0;
            m[j] = i < stretches ? S.table_mass[i] : 0.0;
            eq_to += eq[j];
        }
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t up = __shfl_up_sync(kFull, eq_to, o);
            if (lane >= o) eq_to += up;
        }
        uint32_t before = eq_to;
#pragma unroll
        for (uint32_t j = 0; j < STRETCHES; ++j) before -= eq[j];
        const uint32_t equal_from = before;
        if (infinite && !first_only) {
            const uint32_t all_equal = __shfl_sync(kFull, eq_to, 31);
            ties = by_count ? min((uint32_t)k_given, all_equal) : all_equal;
            if (by_mass) ties = max(1u, min(ties, (uint32_t)ceil((double)p * ties)));
        }
#pragma unroll
        for (uint32_t j = 0; j < STRETCHES; ++j) {
            m[j] += (double)(before < ties ? min(eq[j], ties - before) : 0) * cut_weight;
            before += eq[j];
            m_to += m[j];
        }
        const double own = m_to;
        for (int o = 1; o < 32; o <<= 1) {
            const double up = __shfl_up_sync(kFull, m_to, o);
            if (lane >= o) m_to += up;
        }
        const double all = __shfl_sync(kFull, m_to, 31), aim = fmin(fmax((double)u, 0.0), 1.0) * all;
        const uint32_t over = __ballot_sync(kFull, own > 0.0 && m_to > aim), some = __ballot_sync(kFull, own > 0.0);
        // (lanes' sums may round so that none exceeds what is drawn, or none of a lane's stretches does: then the last that has a mass)
        if (lane == (over ? __ffs(over) - 1 : 31 - __clz(some | 1u))) {
            double r = m_to - own, from = 0.0;
            uint32_t seen = equal_from, equal = 0, at = lane * STRETCHES;
            bool done = false;
#pragma unroll
            for (uint32_t j = 0; j < STRETCHES; ++j) {
                if (m[j] > 0.0 && !done) from = r, equal = seen, at = lane * STRETCHES + j, done = over && r + m[j] > aim;
                r += m[j];
                seen += eq[j];
            }
            S.draw_stretch = at, S.draw_equal = equal, S.ties = ties, S.draw_from = from, S.draw_aim = done ? aim : INFINITY;
        }
    }
    __syncthreads();
    if (S.draw_stretch / kSampleWarps != rank) return;
    // the stretch's CTA: its warps share it, and the one that has the draw goes through its part
    const uint32_t drawn = S.draw_stretch % kSampleWarps, drawn_from = min(R.pieces, drawn * stretch), drawn_to = min(R.pieces, drawn_from + stretch);
    const uint32_t part = (drawn_to - drawn_from + kSampleWarps * 32 - 1) / (kSampleWarps * 32) * 32;
    uint32_t equal_before = S.draw_equal, from = drawn_from, to = drawn_to;
    double run = S.draw_from;
    const double aim = S.draw_aim;
    ties = S.ties;
    sum_stretch(min(drawn_to, drawn_from + warp * part), min(drawn_to, drawn_from + (warp + 1) * part));
    __syncthreads();
    {
        uint32_t chosen = 0, equal_chosen = equal_before, equal = equal_before;
        double run_chosen = run, r = run;
        bool done = false;
        for (uint32_t w = 0; w < kSampleWarps; ++w) {
            const uint32_t eq = S.warp_equal[w];
            const double m = S.warp_mass[w] + (double)(equal < ties ? min(eq, ties - equal) : 0) * cut_weight;
            if (m > 0.0 && !done) chosen = w, equal_chosen = equal, run_chosen = r, done = r + m > aim;
            r += m;
            equal += eq;
        }
        if (warp != chosen) return;
        equal_before = equal_chosen;
        run = run_chosen;
        from = min(drawn_to, drawn_from + warp * part);
        to = min(drawn_to, from + part);
    }
    int32_t token = -1;
    for (uint32_t i0 = from; i0 < to; i0 += 32) {
        const uint32_t i = i0 + lane;
        const Piece16<TYPE> x(i < to ? R.raw(i) : make_uint4(kFull, kFull, kFull, kFull));
        float w[R.N];
        uint32_t eq = 0, any = 0;
#pragma unroll
        for (int e = 0; e < R.N; ++e) eq += x.x[e] == cut, any |= x.x[e] >= cut;
        if (!__any_sync(kFull, any)) continue;
        uint32_t eq_to = eq;
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t up = __shfl_up_sync(kFull, eq_to, o);
            if (lane >= o) eq_to += up;
        }
        uint32_t seen = equal_before + eq_to - eq;
        double m = 0.0;
#pragma unroll
        for (int e = 0; e < R.N; ++e) {
            w[e] = 0.0f;
            if (x.x[e] > cut) w[e] = weight(x.x[e]);
            if (x.x[e] == cut && seen++ < ties) w[e] = cut_weight;
            m += w[e];
        }
        double m_to = m;
        for (int o = 1; o < 32; o <<= 1) {
            const double up = __shfl_up_sync(kFull, m_to, o);
            if (lane >= o) m_to += up;
        }
        const uint32_t over = __ballot_sync(kFull, m > 0.0 && run + m_to > aim), some = __ballot_sync(kFull, m > 0.0);
        if (some) {
            const int who = over ? __ffs(over) - 1 : 31 - __clz(some);
            if (lane == who) {
                double r = run + m_to - m;
                int e = -1;
#pragma unroll
                for (int j = 0; j < R.N; ++j) {
                    const bool was_over = e >= 0 && r > aim;
                    if (w[j] > 0.0f && !was_over) {
                        r += w[j];
                        e = j;
                    }
                }
                token = (int32_t)(i * R.N + e) - (int32_t)R.phase;
            }
            token = __shfl_sync(kFull, token, who);
            if (over) break;
        }
        equal_before += __shfl_sync(kFull, eq_to, 31);
        run += __shfl_sync(kFull, m_to, 31);
    }
    if (lane == 0) A.tokens[row] = (int32_t)i0 + token;
}

template <int TYPE>
static cudaError_t launch_type(const SamplingArgs &a, uint32_t ctas, uint32_t smem, cudaStream_t stream) {
    static std::atomic<bool> attr_set[64];             // set twice by racing threads at worst: the call is idempotent
    int dev = 0;
    cudaGetDevice(&dev);
    if (dev < 0 || dev >= 64 || !attr_set[dev].load(std::memory_order_acquire)) {
        const cudaError_t e = cudaFuncSetAttribute(sample_kernel<TYPE>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSampleMostSmem);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) attr_set[dev].store(true, std::memory_order_release);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(a.rows * ctas);
    cfg.blockDim = dim3(kSampleThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ctas;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, sample_kernel<TYPE>, a);
}

cudaError_t launch_sampling(const SamplingArgs &args, uint32_t sms, cudaStream_t stream) {
    SamplingArgs a = args;
    const uint32_t size = a.type == 0 ? 4 : 2;
    // As many CTAs a row as keep what all that run together read again and again, 64 MB, in L2; more where that leaves SMs idle and CTAs with
    // more than 2048 logits.  What shared memory has room for stays there.
    const uint64_t slots = (uint64_t)sms * kSampleEach;
    auto running = [&](uint64_t n) { return a.rows * n < slots ? a.rows * n : slots; };
    uint32_t ctas = 1;
    while (ctas < kMostCluster && (running(ctas) * ((uint64_t)a.vocab * size / ctas) > (64ull << 20) || (a.rows * (uint64_t)ctas * 2 <= slots && a.vocab > ctas * 2048u))) ctas *= 2;
    a.part = (uint32_t)(((uint64_t)a.vocab + ctas - 1) / ctas);
    const uint64_t each = (running(ctas) + sms - 1) / sms;             // CTAs of an SM
    const uint64_t pieces = ((uint64_t)a.part * size + 30) / 16, all = kSampleMostSmem / each - (each > 1 ? 1024 : 0);
    const uint64_t room = all > sizeof(SampleShared) ? (all - sizeof(SampleShared)) / 16 : 0;
    a.kept_pieces = (uint32_t)(pieces < room ? pieces : room);
    const uint32_t smem = (uint32_t)sizeof(SampleShared) + a.kept_pieces * 16;
    return a.type == 0 ? launch_type<0>(a, ctas, smem, stream) : a.type == 1 ? launch_type<1>(a, ctas, smem, stream) : launch_type<2>(a, ctas, smem, stream);
}

}  // namespace huffllm
