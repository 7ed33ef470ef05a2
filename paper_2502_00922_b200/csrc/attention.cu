// Attention over the 4-bit cache: one pass over the visible tokens with the running maximum and sum of the softmax.
#include <cuda_runtime.h>

#include "cache_rows.cuh"
#include "decode_common.cuh"
#include "epilogue.cuh"

namespace huffllm {

constexpr uint32_t kAttentionWarps = 4;

// A CTA per row and query head; its warps take every fourth token, a lane has channel `lane` of each group.
template <bool F16>
__global__ void __launch_bounds__(kAttentionWarps * 32) attention_kernel(const __grid_constant__ AttentionArgs A) {
    constexpr int G = 8;
    __shared__ float s_max[kAttentionWarps], s_sum[kAttentionWarps], s_acc[kAttentionWarps][G * 32];
    pdl_launch_dependents();
    pdl_wait_prior_grid();
    const CacheArgs &C = A.c;
    const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, row = blockIdx.x, head = blockIdx.y, groups = cache_groups(C.dim);
    if (row == 0 && head == 0) report_faults(C, A.starts, A.rows, A.err);
    const uint32_t b = sequence_of_row(A.starts, C.sequences, row);
    if (b >= C.sequences) return;
    const Sequence S = sequence_of(C, A.starts, A.rows, b);
    if (row < S.first_row || row - S.first_row >= S.rows) return;
    const int32_t at = S.tokens - (int32_t)S.rows + (int32_t)(row - S.first_row);
    float q[G], acc[G], top = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int g = 0; g < G; ++g) {
        q[g] = g < groups ? widen16<F16>(__ldcg(A.q + row * A.q_stride + head * C.dim + g * 32 + lane)) * A.scale : 0.0f;
        acc[g] = 0.0f;
    }
    const uint32_t t = lane / 8, shift = (lane & 1) * 16 + (lane % 8 >> 1) * 4;
    for (int32_t j = warp; j <= at; j += kAttentionWarps) {
        if (A.window && j <= at - (int64_t)A.window && (uint32_t)j >= A.sinks) continue;
        const uint8_t *const block = block_of(C, b, j, head / A.group);
        if (!block) {
            if (A.err && lane == 0) *A.err = (int32_t)b + 1;
            continue;
        }
        const uint32_t r = j % kCacheBlock;
        float dot = 0.0f;
#pragma unroll
        for (int g = 0; g < G; ++g)
            if (g < groups) {
                const uint32_t code = *(const uint32_t *)(block + key_word_at(C.dim, r, g, t)) >> shift & 15u;
                const float s = __half2float(*(const __half *)(block + key_scale_at(C.dim, r, g))), m = __half2float(*(const __half *)(block + key_offset_at(C.dim, r, g)));
                dot = fmaf(q[g], fmaf(s, (float)code, m), dot);
            }
        for (int o = 16; o; o >>= 1) dot += __shfl_xor_sync(0xFFFFFFFFu, dot, o);
        const float next = fmaxf(top, dot), keep = top == -INFINITY ? 0.0f : expf(top - next), p = dot == -INFINITY ? 0.0f : expf(dot - next);
        top = next;
        sum = fmaf(sum, keep, p);
#pragma unroll
        for (int g = 0; g < G; ++g)
            if (g < groups) {
                const uint32_t d = g * 32 + lane, code = block[value_byte_at(C.dim, r, lane % 16 < 8 ? d : d - 8)] >> (lane % 16 < 8 ? 0 : 4) & 15u;
                const float s = __half2float(*(const __half *)(block + value_scale_at(C.dim, r, g))), m = __half2float(*(const __half *)(block + value_offset_at(C.dim, r, g)));
                acc[g] = fmaf(acc[g], keep, p * fmaf(s, (float)code, m));
            }
    }
    if (lane == 0) s_max[warp] = top, s_sum[warp] = sum;
#pragma unroll
    for (int g = 0; g < G; ++g) s_acc[warp][g * 32 + lane] = acc[g];
    __syncthreads();
    float all = -INFINITY, total = 0.0f, keep[kAttentionWarps];
    for (int w = 0; w < kAttentionWarps; ++w) all = fmaxf(all, s_max[w]);
    for (int w = 0; w < kAttentionWarps; ++w) {
        keep[w] = s_max[w] == -INFINITY ? (s_sum[w] != s_sum[w] ? s_sum[w] : 0.0f) : expf(s_max[w] - all);
        total += keep[w] * s_sum[w];
    }
    for (uint32_t d = threadIdx.x; d < C.dim; d += kAttentionWarps * 32) {
        float o = 0.0f;
        for (int w = 0; w < kAttentionWarps; ++w) o += keep[w] * s_acc[w][d];
        A.out[row * A.out_stride + head * C.dim + d] = round16<F16>(total == 0.0f ? 0.0f : o / total);
    }
}

cudaError_t launch_attention(const AttentionArgs &a, uint32_t, cudaStream_t stream) {
    return launch_behind(a.c.fp16 ? attention_kernel<true> : attention_kernel<false>, dim3(a.rows, a.heads), kAttentionWarps * 32, 0, stream, a);
}

}  // namespace huffllm
