// Launch interface of the operators between and behind a decode step's products: rotary positions, the 4-bit cache and its attention,
// sampling.
#pragma once
#include <cuda_runtime.h>
#include <atomic>
#include <cstdint>

namespace huffllm {

// Strides in values, never 0; fp16: 16-bit values are FP16 (else BF16).
struct RotaryArgs {
    const int32_t *positions;
    const float *frequencies;
    const uint16_t *in[2];         // q, k
    uint16_t *out[2];
    uint64_t in_stride[2], out_stride[2];
    uint32_t heads[2];
    uint32_t tokens, dim, rot, neighbours, fp16;
    uint32_t axis_bits[32];        // the axis of every pair, two bits each
};
cudaError_t launch_rotary(const RotaryArgs &a, cudaStream_t stream);

struct CacheArgs {
    uint8_t *pool;
    const int32_t *table, *lengths;
    uint32_t pages, kv_heads, dim, page_tokens, sequences, table_stride, fp16;
};
struct CacheRows {
    uint16_t *k, *v;               // append: only read; read: fp32 or 16 bits
    uint64_t k_stride, v_stride;
    const int32_t *starts;         // may be null
    uint32_t rows;
    uint32_t f32;                  // read: k and v are fp32
    int32_t *err;                  // may be null
};
cudaError_t launch_cache_append(const CacheArgs &c, const CacheRows &r, cudaStream_t stream);
cudaError_t launch_cache_read(const CacheArgs &c, const CacheRows &r, cudaStream_t stream);

constexpr uint32_t kAttentionCtas = 512;                  // most CTAs of a launch
constexpr uint32_t kAttentionPartial = 16 * 132;          // most floats of a piece (a column's channels and four more: 16 columns of 128, eight of 256)
struct AttentionArgs {
    CacheArgs c;
    const uint16_t *q;
    uint16_t *out;
    uint64_t q_stride, out_stride;
    const int32_t *starts;         // may be null
    uint32_t rows, heads, group;   // group: query heads of a key head
    uint32_t window, sinks;
    uint32_t page_recip;           // floor(2^32 / blocks of a page) (one block: less one)
    float scale;
    int32_t *err;                  // may be null
    unsigned int *tickets;         // zero between calls
    float *partials;               // two pieces a CTA
};
cudaError_t launch_attention(const AttentionArgs &a, uint32_t sms, cudaStream_t stream);

constexpr uint32_t kSampleMostSmem = 227 * 1024;
struct SamplingArgs {
    const void *logits;
    uint64_t stride;
    const float *temperature;      // the settings may be null
    const int32_t *top_k;
    const float *top_p, *min_p, *uniform;
    int32_t *tokens;
    uint32_t rows, vocab, type;    // type 0: fp32, 1: BF16, 2: FP16
    uint32_t part, kept_pieces;    // (the launcher's) logits of a CTA; how many 16-byte pieces of them it keeps in shared memory
};
cudaError_t launch_sampling(const SamplingArgs &a, uint32_t sms, cudaStream_t stream);

// A launch whose set-up may overlap the tail of the kernel in front of it.
template <typename... Params, typename... Args>
cudaError_t launch_behind(void (*kernel)(Params...), dim3 grid, uint32_t threads, uint32_t smem, cudaStream_t stream, const Args &...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
}

}  // namespace huffllm
