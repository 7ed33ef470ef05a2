// The next token of a row of logits, from a given random number.
//
// What stays is a beginning of the order (largest logit first, lower index first among equals), so it is told by its last logit's key and
// by how many of those with that very key stay.  Both cuts (top_k by number, top_p by mass) are found by halving the keys' range.
#include <cuda_runtime.h>

#include "decode_common.cuh"
#include "decode_step.h"
#include "epilogue.cuh"

namespace huffllm {

constexpr uint32_t kSampleThreads = 1024;

// Ascending with the value; NaN and minus infinity lowest, both zeros alike.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t u = __float_as_uint(x == 0.0f ? 0.0f : x);
    return x != x ? 0x007FFFFFu : u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key); }
constexpr uint32_t kLowestKey = 0x007FFFFFu;

template <int TYPE>
__device__ __forceinline__ float logit_at(const void *p, uint64_t i) {
    if (TYPE == 0) return __ldcg((const float *)p + i);
    return widen16<TYPE == 2>(__ldcg((const unsigned short *)p + i));
}

template <typename T, typename Op>
__device__ T block_reduce(T v, Op op, T *scratch) {
    const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    for (int o = 16; o; o >>= 1) v = op(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    __syncthreads();
    if (lane == 0) scratch[warp] = v;
    __syncthreads();
    v = scratch[lane];
    for (int o = 16; o; o >>= 1) v = op(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
}

template <int TYPE>
__global__ void __launch_bounds__(kSampleThreads) sample_kernel(const __grid_constant__ SamplingArgs A) {
    __shared__ double s_d[32];
    __shared__ uint32_t s_u[32];
    __shared__ double s_part[kSampleThreads];
    pdl_launch_dependents();
    pdl_wait_prior_grid();
    const uint32_t tid = threadIdx.x, row = blockIdx.x, n = A.vocab;
    const uint64_t base = row * A.stride;
    const float t = A.temperature ? __ldcg(A.temperature + row) : 1.0f;
    const bool greedy = !(t > 0.0f);
    const float u = __ldcg(A.uniform + row), top_p = A.top_p ? __ldcg(A.top_p + row) : 1.0f, given = A.min_p ? __ldcg(A.min_p + row) : 0.0f, least = given > 1.0f ? 1.0f : given;
    const int32_t k = greedy ? 1 : A.top_k ? __ldcg(A.top_k + row) : 0;
    auto add_u = [](uint32_t a, uint32_t b) { return a + b; };
    auto add_d = [](double a, double b) { return a + b; };
    auto max_u = [](uint32_t a, uint32_t b) { return max(a, b); };
    uint32_t top = 0;
    for (uint32_t i = tid; i < n; i += kSampleThreads) top = max(top, key_of(logit_at<TYPE>(A.logits, base + i)));
    top = block_reduce(top, max_u, s_u);
    if (top <= kLowestKey) {
        if (tid == 0) A.tokens[row] = -1;
        return;
    }
    const float most = value_of(top);
    auto weight = [&](uint32_t key) -> float { return key == top ? 1.0f : greedy || most == INFINITY ? 0.0f : expf((value_of(key) - most) / t); };
    auto key_at = [&](uint32_t i) { return key_of(logit_at<TYPE>(A.logits, base + i)); };
    // how many keys (and what mass) are above `cut`
    auto above = [&](uint32_t cut, double *mass) -> uint32_t {
        uint32_t c = 0;
        double m = 0.0;
        for (uint32_t i = tid; i < n; i += kSampleThreads) {
            const uint32_t key = key_at(i);
            if (key > cut) {
                ++c;
                m += weight(key);
            }
        }
        c = block_reduce(c, add_u, s_u);
        *mass = block_reduce(m, add_d, s_d);
        return c;
    };
    // the cut: keys above `cut` stay, and `ties` of those that equal it
    uint32_t cut = kLowestKey, ties = 0;
    double mass;
    uint32_t count = above(cut, &mass);
    if (k > 0 && (uint32_t)k < count) {
        uint32_t lo = kLowestKey, hi = top;              // fewer than k above hi, k or more above lo
        while (hi - lo > 1) {
            const uint32_t mid = lo + (hi - lo) / 2;
            if (above(mid, &mass) < (uint32_t)k) hi = mid;
            else lo = mid;
        }
        cut = hi;
        ties = (uint32_t)k - above(cut, &mass);
        mass += (double)ties * weight(cut);
    }
    if (top_p < 1.0f) {
        const double want = fmax((double)top_p, 0.0) * mass;
        uint32_t lo = cut, hi = top;                     // less than `want` above hi; `want` or more above lo, or lo is the cut
        double m;
        while (hi - lo > 1) {
            const uint32_t mid = lo + (hi - lo) / 2;
            above(mid, &m);
            if (m < want) hi = mid;
            else lo = mid;
        }
        above(lo, &m);
        const bool at_cut = lo == cut && m < want;       // (the cut's own ties are needed too)
        const uint32_t edge = at_cut ? cut : hi;
        const uint32_t over = above(edge, &m), at = at_cut ? ties : above(edge - 1, &mass) - over;
        const double each = weight(edge), left = want - m;
        const double need = each > 0.0 ? ceil(left / each) : (double)at;
        cut = edge;
        ties = (uint32_t)fmin(fmax(need, over ? 0.0 : 1.0), (double)at);
    }
    // the draw, in the order of indexes: a thread's share follows the one before
    const uint32_t share = (n + kSampleThreads - 1) / kSampleThreads, from = min(n, tid * share), to = min(n, from + share);
    uint32_t equal = 0;
    for (uint32_t i = from; i < to; ++i) equal += key_at(i) == cut;
    s_part[tid] = equal;
    __syncthreads();
    uint32_t before = 0;
    for (uint32_t i = 0; i < tid; ++i) before += (uint32_t)s_part[i];
    __syncthreads();
    auto stays = [&](uint32_t key, uint32_t &seen) -> double {
        const bool in = key > cut || (key == cut && seen++ < ties);
        const float w = in ? weight(key) : 0.0f;
        return w < least ? 0.0 : (double)w;
    };
    double part = 0.0;
    uint32_t seen = before;
    for (uint32_t i = from; i < to; ++i) part += stays(key_at(i), seen);
    s_part[tid] = part;
    __syncthreads();
    double total = 0.0, ahead = 0.0;
    for (uint32_t i = 0; i < kSampleThreads; ++i) {
        if (i == tid) ahead = total;
        total += s_part[i];
    }
    const double aim = fmin(fmax((double)u, 0.0), 1.0) * total;
    if (part > 0.0) {
        double run = ahead;
        int32_t found = -1, last = -1;
        seen = before;
        for (uint32_t i = from; i < to && found < 0; ++i) {
            const double w = stays(key_at(i), seen);
            if (w > 0.0) last = (int32_t)i;
            run += w;
            if (w > 0.0 && run > aim) found = (int32_t)i;
        }
        if (found >= 0 && ahead <= aim) A.tokens[row] = found;
        if (found < 0 && ahead + part >= total && aim >= total) A.tokens[row] = last;
    }
}

cudaError_t launch_sampling(const SamplingArgs &a, uint32_t, cudaStream_t stream) {
    return launch_behind(a.type == 0 ? sample_kernel<0> : a.type == 1 ? sample_kernel<1> : sample_kernel<2>, dim3(a.rows), kSampleThreads, 0, stream, a);
}

}  // namespace huffllm
