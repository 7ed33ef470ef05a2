// The 4-bit cache: new tokens written, tokens read back.
#include <cuda_runtime.h>

#include "cache_rows.cuh"
#include "decode_common.cuh"
#include "epilogue.cuh"

namespace huffllm {

constexpr uint32_t kCacheThreads = 256;

// Scale and offset of a group from its smallest and largest value; false where it stands for NaN.
__device__ __forceinline__ bool scale_of(float low, float high, bool finite, __half &s, __half &m) {
    s = __float2half_rn(__fdiv_rn(high - low, 15.0f));
    m = __float2half_rn(low);
    if (finite && __half2float(s) < INFINITY && fabsf(__half2float(m)) < INFINITY) return true;
    s = __ushort_as_half(0x7FFFu);
    m = __ushort_as_half(0u);
    return false;
}
// The code of x: (x - m) / s, exactly rounded.  The quotient in fp32 is off by less than 1e-5, so 64 bits decide only next to a border.
__device__ __forceinline__ uint32_t code_of(float x, float s, float m) {
    if (s == 0.0f) return 0;
    float q = (x - m) / s;
    if (fabsf(q - floorf(q) - 0.5f) < 1e-4f) q = (float)rint(((double)x - (double)m) / (double)s);
    return (uint32_t)fminf(fmaxf(rintf(q), 0.0f), 15.0f);
}

// A warp per row, head and side (keys, values); a lane has channel `lane` of a group.
template <bool F16>
__global__ void __launch_bounds__(kCacheThreads) cache_append_kernel(const __grid_constant__ CacheArgs C, const __grid_constant__ CacheRows R) {
    pdl_launch_dependents();
    pdl_wait_prior_grid();
    if (blockIdx.x == 0) report_faults(C, R.starts, R.rows, R.err);
    const uint32_t lane = threadIdx.x % 32;
    const uint64_t item = (uint64_t)blockIdx.x * (kCacheThreads / 32) + threadIdx.x / 32;
    const uint32_t row = (uint32_t)(item / (2 * C.kv_heads)), h = (uint32_t)(item % (2 * C.kv_heads)) / 2, side = item % 2;
    if (row >= R.rows) return;
    const uint32_t b = sequence_of_row(R.starts, C.sequences, row);
    if (b >= C.sequences) return;
    const Sequence S = sequence_of(C, R.starts, R.rows, b);
    if (S.bad || row < S.first_row || row - S.first_row >= S.rows) return;
    const int32_t at = S.tokens - (int32_t)S.rows + (int32_t)(row - S.first_row);
    if (at < 0) return;
    uint8_t *const block = block_of(C, b, at, h);
    if (!block) {
        if (R.err && lane == 0) *R.err = (int32_t)b + 1;
        return;
    }
    const uint32_t r = at % kCacheBlock;
    const uint16_t *x = (side ? R.v + row * R.v_stride : R.k + row * R.k_stride) + h * C.dim;
    for (uint32_t g = 0; g < cache_groups(C.dim); ++g) {
        const float v = widen16<F16>(__ldcg(x + g * kCacheGroup + lane));
        float low = v, high = v;
        for (int o = 16; o; o >>= 1) {
            low = fminf(low, __shfl_xor_sync(0xFFFFFFFFu, low, o));
            high = fmaxf(high, __shfl_xor_sync(0xFFFFFFFFu, high, o));
        }
        __half s, m;
        const bool sound = scale_of(low, high, __all_sync(0xFFFFFFFFu, fabsf(v) < INFINITY), s, m);
        const uint32_t code = sound ? code_of(v, __half2float(s), __half2float(m)) : 0u;
        if (side == 0) {
            uint32_t word = code << ((lane & 1) * 16 + (lane % 8 >> 1) * 4);
            for (int o = 1; o < 8; o <<= 1) word |= __shfl_xor_sync(0xFFFFFFFFu, word, o);
            if (lane % 8 == 0) *(uint32_t *)(block + key_word_at(C.dim, r, g, lane / 8)) = word;
        } else {
            const uint32_t other = __shfl_xor_sync(0xFFFFFFFFu, code, 8);
            if (lane % 16 < 8) block[value_byte_at(C.dim, r, g * kCacheGroup + lane)] = (uint8_t)(code | other << 4);
        }
        if (lane == 0) {
            *(__half *)(block + (side ? value_scale_at(C.dim, r, g) : key_scale_at(C.dim, r, g))) = s;
            *(__half *)(block + (side ? value_offset_at(C.dim, r, g) : key_offset_at(C.dim, r, g))) = m;
            // (keys' offsets are read in pairs, and what is read is multiplied by 0: it must be a number)
            if (side == 0 && g + 1 == cache_groups(C.dim) && g % 2 == 0) *(__half *)(block + key_offset_at(C.dim, r, g + 1)) = __ushort_as_half(0);
        }
    }
}

template <bool F16>
__global__ void __launch_bounds__(kCacheThreads) cache_read_kernel(const __grid_constant__ CacheArgs C, const __grid_constant__ CacheRows R) {
    pdl_launch_dependents();
    pdl_wait_prior_grid();
    if (blockIdx.x == 0) report_faults(C, R.starts, R.rows, R.err);
    const uint32_t lane = threadIdx.x % 32;
    const uint64_t item = (uint64_t)blockIdx.x * (kCacheThreads / 32) + threadIdx.x / 32;
    const uint32_t row = (uint32_t)(item / (2 * C.kv_heads)), h = (uint32_t)(item % (2 * C.kv_heads)) / 2, side = item % 2;
    if (row >= R.rows) return;
    const uint32_t b = sequence_of_row(R.starts, C.sequences, row);
    if (b >= C.sequences) return;
    const Sequence S = sequence_of(C, R.starts, R.rows, b);
    if (S.bad || row < S.first_row || row - S.first_row >= S.rows) return;
    const int32_t at = S.tokens - (int32_t)S.rows + (int32_t)(row - S.first_row);
    if (at < 0) return;
    const uint8_t *const block = block_of(C, b, at, h);
    if (!block) {
        if (R.err && lane == 0) *R.err = (int32_t)b + 1;
        return;
    }
    const uint32_t r = at % kCacheBlock;
    void *const out = side ? (void *)R.v : (void *)R.k;
    if (!out) return;
    const uint64_t to = row * (side ? R.v_stride : R.k_stride) + h * C.dim;
    for (uint32_t g = 0; g < cache_groups(C.dim); ++g) {
        const uint32_t d = g * kCacheGroup + lane;
        uint32_t code;
        if (side == 0) code = *(const uint32_t *)(block + key_word_at(C.dim, r, g, lane / 8)) >> ((lane & 1) * 16 + (lane % 8 >> 1) * 4) & 15u;
        else code = block[value_byte_at(C.dim, r, lane % 16 < 8 ? d : d - 8)] >> (lane % 16 < 8 ? 0 : 4) & 15u;
        const float s = __half2float(*(const __half *)(block + (side ? value_scale_at(C.dim, r, g) : key_scale_at(C.dim, r, g))));
        const float m = __half2float(*(const __half *)(block + (side ? value_offset_at(C.dim, r, g) : key_offset_at(C.dim, r, g))));
        const float v = fmaf(s, (float)code, m);
        if (R.f32) ((float *)out)[to + d] = v;
        else ((uint16_t *)out)[to + d] = round16<F16>(v);
    }
}

static uint32_t items_grid(const CacheArgs &c, const CacheRows &r) {
    const uint64_t warps = (uint64_t)r.rows * c.kv_heads * 2;
    return (uint32_t)((warps + kCacheThreads / 32 - 1) / (kCacheThreads / 32));
}
cudaError_t launch_cache_append(const CacheArgs &c, const CacheRows &r, uint32_t, cudaStream_t stream) {
    return launch_behind(c.fp16 ? cache_append_kernel<true> : cache_append_kernel<false>, dim3(items_grid(c, r)), kCacheThreads, 0, stream, c, r);
}
cudaError_t launch_cache_read(const CacheArgs &c, const CacheRows &r, uint32_t, cudaStream_t stream) {
    return launch_behind(c.fp16 ? cache_read_kernel<true> : cache_read_kernel<false>, dim3(items_grid(c, r)), kCacheThreads, 0, stream, c, r);
}

}  // namespace huffllm
