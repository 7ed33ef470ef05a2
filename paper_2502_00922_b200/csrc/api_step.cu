// C-ABI entry points of the operators between and behind a decode step's products: argument checks and launches.
#include <cuda_runtime.h>
#include <cstring>

#include "cache_layout.h"
#include "decode_step.h"
#include "internal.h"

using namespace huffllm;

namespace {

constexpr uint64_t kMost = 0x7FFFFFFFull;

bool aligned(const void *p, uintptr_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// A stride of 0 is packed; false where it is below the values of a row.
bool stride_of(uint64_t given, uint64_t packed, uint64_t *out) {
    *out = given ? given : packed;
    return *out >= packed && *out <= (1ull << 40);
}

// Do rows of `values` 16-bit values each overlap?  Known where the strides are alike, and of the first rows; with other strides rows may lie between rows.
bool rows_overlap(const uint16_t *a, const uint16_t *b, uint64_t values, uint64_t a_stride, uint64_t b_stride, uint64_t rows) {
    const uint64_t apart = (uint64_t)((uintptr_t)a < (uintptr_t)b ? (uintptr_t)b - (uintptr_t)a : (uintptr_t)a - (uintptr_t)b), width = 2 * values;
    if (rows == 1 || a_stride != b_stride) return apart < width;
    const uint64_t step = 2 * a_stride, k = apart / step, left = apart % step;       // the later one's first row lies behind the other's row k, or in front of its row k + 1
    return (k < rows && left < width) || (k + 1 < rows && step - left < width);
}

huffllm_status check_cache(const huffllm_cache *c, bool pool) {
    if (!c) return fail(HUFFLLM_ERR_INVALID_ARG, "null pointer");
    if (c->dtype > HUFFLLM_FP16) return fail(HUFFLLM_ERR_INVALID_ARG, "unknown type");
    if (c->kv_heads == 0 || c->pages == 0) return fail(HUFFLLM_ERR_INVALID_ARG, "kv_heads and pages must be at least 1");
    if (c->head_dim != 64 && c->head_dim != 96 && c->head_dim != 128 && c->head_dim != 192 && c->head_dim != 256)
        return fail(HUFFLLM_ERR_UNSUPPORTED, "head_dim %u is not 64, 96, 128, 192 or 256", c->head_dim);
    if (c->page_tokens == 0 || c->page_tokens % kCacheBlock || c->page_tokens > 65536)
        return fail(HUFFLLM_ERR_INVALID_ARG, "page_tokens must be a multiple of %u, at most 65536", kCacheBlock);
    if (c->kv_heads > 4096) return fail(HUFFLLM_ERR_UNSUPPORTED, "at most 4096 key heads");
    if (c->pages > kMost) return fail(HUFFLLM_ERR_UNSUPPORTED, "at most 2^31 - 1 pages");
    if (!pool) return HUFFLLM_OK;
    if (!c->pool || !c->table || !c->lengths) return fail(HUFFLLM_ERR_INVALID_ARG, "null pointer");
    if (!aligned(c->pool, 256) || !aligned(c->table, 4) || !aligned(c->lengths, 4))
        return fail(HUFFLLM_ERR_INVALID_ARG, "pool must be 256-byte, table and lengths 4-byte aligned");
    if (c->sequences == 0 || c->table_stride == 0) return fail(HUFFLLM_ERR_INVALID_ARG, "sequences and table_stride must be at least 1");
    if (c->sequences > (1u << 20)) return fail(HUFFLLM_ERR_UNSUPPORTED, "at most 2^20 sequences");
    return HUFFLLM_OK;
}

// Rows of a call: without starts every sequence has one.
huffllm_status check_rows(const huffllm_cache &c, uint64_t rows, const int32_t *starts, const int32_t *err) {
    if (rows == 0) return fail(HUFFLLM_ERR_INVALID_ARG, "rows must be at least 1");
    if (rows > (1ull << 24)) return fail(HUFFLLM_ERR_UNSUPPORTED, "at most 2^24 rows per call");
    if (!starts && rows != c.sequences) return fail(HUFFLLM_ERR_INVALID_ARG, "without starts there is one row per sequence: %u, not %llu", c.sequences, (unsigned long long)rows);
    if (!aligned(starts, 4) || !aligned(err, 4)) return fail(HUFFLLM_ERR_INVALID_ARG, "starts and err_flag must be aligned to their types");
    return HUFFLLM_OK;
}

CacheArgs cache_args(const huffllm_cache &c) {
    CacheArgs a;
    memset(&a, 0, sizeof(a));
    a.pool = (uint8_t *)c.pool;
    a.table = c.table;
    a.lengths = c.lengths;
    a.pages = (uint32_t)c.pages;
    a.kv_heads = c.kv_heads;
    a.dim = c.head_dim;
    a.page_tokens = c.page_tokens;
    a.sequences = c.sequences;
    a.table_stride = c.table_stride;
    a.fp16 = c.dtype == HUFFLLM_FP16;
    return a;
}

huffllm_status launched(cudaError_t e, const char *what) {
    return e == cudaSuccess ? HUFFLLM_OK : fail(HUFFLLM_ERR_CUDA, "%s launch: %s", what, cudaGetErrorString(e));
}

}  // namespace

extern "C" {

huffllm_status huffllm_apply_rotary(const huffllm_rotary *args, huffllm_stream stream) {
    clear_error();
    if (!args) return fail(HUFFLLM_ERR_INVALID_ARG, "null pointer");
    const huffllm_rotary &a = *args;
    if (!a.q || !a.q_out || (a.k != nullptr) != (a.k_out != nullptr) || !a.positions || !a.frequencies) return fail(HUFFLLM_ERR_INVALID_ARG, "null pointer");
    if (a.dtype > HUFFLLM_FP16 || a.pairing > HUFFLLM_PAIR_NEIGHBOURS) return fail(HUFFLLM_ERR_INVALID_ARG, "unknown type or pairing");
    if (a.tokens == 0 || a.q_heads == 0 || (a.k && a.k_heads == 0)) return fail(HUFFLLM_ERR_INVALID_ARG, "tokens and heads must be at least 1");
    if (a.rotary_dim == 0 || a.rotary_dim % 2 || a.rotary_dim > a.head_dim) return fail(HUFFLLM_ERR_INVALID_ARG, "rotary_dim must be even, and at most head_dim");
    if (a.axes == 0 || a.axes > HUFFLLM_MAX_AXES) return fail(HUFFLLM_ERR_INVALID_ARG, "1 to %d axes", HUFFLLM_MAX_AXES);
    uint64_t pairs = 0;
    for (uint32_t i = 0; i < a.axes; ++i) pairs += a.sections[i];
    if (pairs != a.rotary_dim / 2) return fail(HUFFLLM_ERR_INVALID_ARG, "sections must add up to rotary_dim / 2");
    if (a.head_dim > 1024 || a.q_heads > 4096 || (a.k && a.k_heads > 4096) || a.tokens > (1ull << 24))
        return fail(HUFFLLM_ERR_UNSUPPORTED, "at most 1024 channels, 4096 heads and 2^24 tokens per call");
    for (const void *p : {(const void *)a.q, (const void *)a.k, (const void *)a.q_out, (const void *)a.k_out})
        if (!aligned(p, 2)) return fail(HUFFLLM_ERR_INVALID_ARG, "pointers must be aligned to their types");
    if (!aligned(a.positions, 4) || !aligned(a.frequencies, 4)) return fail(HUFFLLM_ERR_INVALID_ARG, "pointers must be aligned to their types");
    RotaryArgs r;
    memset(&r, 0, sizeof(r));
    r.heads[0] = a.q_heads;
    r.heads[1] = a.k ? a.k_heads : 0;
    const uint64_t q_row = (uint64_t)a.q_heads * a.head_dim, k_row = (uint64_t)r.heads[1] * a.head_dim;
    if (!stride_of(a.q_stride, q_row, &r.in_stride[0]) || !stride_of(a.q_out_stride, q_row, &r.out_stride[0]) ||
        (a.k && (!stride_of(a.k_stride, k_row, &r.in_stride[1]) || !stride_of(a.k_out_stride, k_row, &r.out_stride[1]))))
        return fail(HUFFLLM_ERR_INVALID_ARG, "stride below the values of a token (or above 2^40)");
    if ((a.q == a.q_out && r.in_stride[0] != r.out_stride[0]) || (a.k && a.k == a.k_out && r.in_stride[1] != r.out_stride[1]))
        return fail(HUFFLLM_ERR_INVALID_ARG, "an out in place of its input takes its stride");
    r.positions = a.positions;
    r.frequencies = a.frequencies;
    r.in[0] = a.q;
    r.in[1] = a.k;
    r.out[0] = a.q_out;
    r.out[1] = a.k_out;
    r.tokens = (uint32_t)a.tokens;
    r.dim = a.head_dim;
    r.rot = a.rotary_dim;
    r.neighbours = a.pairing == HUFFLLM_PAIR_NEIGHBOURS;
    r.fp16 = a.dtype == HUFFLLM_FP16;
    // the axis of every pair: one axis behind the other, or dealt in turn to those that have pairs left
    uint32_t left[HUFFLLM_MAX_AXES] = {}, axis = 0;
    for (uint32_t i = 0; i < a.axes; ++i) left[i] = a.sections[i];
    for (uint32_t i = 0; i < a.rotary_dim / 2; ++i) {
        while (left[axis] == 0) axis = (axis + 1) % a.axes;
        r.axis_bits[i / 16] |= axis << i % 16 * 2;
        --left[axis];
        if (a.in_turn) axis = (axis + 1) % a.axes;
    }
    return launched(launch_rotary(r, (cudaStream_t)stream), "rotary");
}

huffllm_status huffllm_cache_bytes(const huffllm_cache *cache, size_t *bytes) {
    clear_error();
    if (!bytes) return fail(HUFFLLM_ERR_INVALID_ARG, "bytes is null");
    const huffllm_status st = check_cache(cache, false);
    if (st != HUFFLLM_OK) return st;
    const uint64_t page = (uint64_t)cache->kv_heads * (cache->page_tokens / kCacheBlock) * cache_block_bytes(cache->head_dim);
    if (cache->pages > (1ull << 62) / page) return fail(HUFFLLM_ERR_UNSUPPORTED, "a cache of 2^62 bytes or more");
    *bytes = cache->pages * page;
    return HUFFLLM_OK;
}

static huffllm_status cache_move(bool append, const huffllm_cache *cache, void *k, void *v, uint32_t type, uint64_t k_stride, uint64_t v_stride,
                                 uint64_t rows, const int32_t *starts, int32_t *err, huffllm_stream stream) {
    clear_error();
    huffllm_status st = check_cache(cache, true);
    if (st != HUFFLLM_OK || (st = check_rows(*cache, rows, starts, err)) != HUFFLLM_OK) return st;
    if (append ? !k || !v : !k && !v) return fail(HUFFLLM_ERR_INVALID_ARG, "null pointer");
    if (type > HUFFLLM_ELEM_16) return fail(HUFFLLM_ERR_INVALID_ARG, "unknown type");
    if (!aligned(k, type == HUFFLLM_ELEM_16 ? 2 : 4) || !aligned(v, type == HUFFLLM_ELEM_16 ? 2 : 4))
        return fail(HUFFLLM_ERR_INVALID_ARG, "pointers must be aligned to their types");
    CacheRows r;
    memset(&r, 0, sizeof(r));
    const uint64_t row = (uint64_t)cache->kv_heads * cache->head_dim;
    if (!stride_of(k_stride, row, &r.k_stride) || !stride_of(v_stride, row, &r.v_stride))
        return fail(HUFFLLM_ERR_INVALID_ARG, "stride below the values of a row (or above 2^40)");
    r.k = (uint16_t *)k;
    r.v = (uint16_t *)v;
    r.starts = starts;
    r.rows = (uint32_t)rows;
    r.f32 = type == HUFFLLM_ELEM_F32;
    r.err = err;
    const CacheArgs c = cache_args(*cache);
    return launched(append ? launch_cache_append(c, r, (cudaStream_t)stream) : launch_cache_read(c, r, (cudaStream_t)stream),
                    append ? "cache append" : "cache read");
}

huffllm_status huffllm_cache_append(const huffllm_cache *cache, const uint16_t *k, const uint16_t *v, uint64_t k_stride, uint64_t v_stride,
                                    uint64_t rows, const int32_t *starts, int32_t *err_flag, huffllm_stream stream) {
    return cache_move(true, cache, (void *)k, (void *)v, HUFFLLM_ELEM_16, k_stride, v_stride, rows, starts, err_flag, stream);
}
huffllm_status huffllm_cache_read(const huffllm_cache *cache, void *k, void *v, uint32_t type, uint64_t k_stride, uint64_t v_stride, uint64_t rows,
                                  const int32_t *starts, int32_t *err_flag, huffllm_stream stream) {
    return cache_move(false, cache, k, v, type, k_stride, v_stride, rows, starts, err_flag, stream);
}

static huffllm_status check_attention(const huffllm_cache *cache, const huffllm_attention *a, bool pool) {
    huffllm_status st = check_cache(cache, pool);
    if (st != HUFFLLM_OK) return st;
    if (!a) return fail(HUFFLLM_ERR_INVALID_ARG, "null pointer");
    if (cache->sequences == 0 || cache->sequences > (1u << 20)) return fail(HUFFLLM_ERR_INVALID_ARG, "1 to 2^20 sequences");
    if (a->heads == 0 || a->heads % cache->kv_heads) return fail(HUFFLLM_ERR_INVALID_ARG, "heads must be a multiple of the cache's kv_heads");
    if (a->heads > 4096) return fail(HUFFLLM_ERR_UNSUPPORTED, "at most 4096 heads");
    if ((st = check_rows(*cache, a->rows, a->starts, nullptr)) != HUFFLLM_OK) return st;
    if (a->rows * a->heads > kMost) return fail(HUFFLLM_ERR_UNSUPPORTED, "rows times heads must stay below 2^31");
    return HUFFLLM_OK;
}

huffllm_status huffllm_attention_control_bytes(const huffllm_cache *cache, const huffllm_attention *args, size_t *bytes) {
    clear_error();
    if (!bytes) return fail(HUFFLLM_ERR_INVALID_ARG, "bytes is null");
    const huffllm_status st = check_attention(cache, args, false);
    if (st != HUFFLLM_OK) return st;
    *bytes = kAttentionCtas * sizeof(unsigned int);
    return HUFFLLM_OK;
}
huffllm_status huffllm_attention_workspace_bytes(const huffllm_cache *cache, const huffllm_attention *args, size_t *bytes) {
    const huffllm_status st = huffllm_attention_control_bytes(cache, args, bytes);
    if (st == HUFFLLM_OK) *bytes += (size_t)kAttentionCtas * 2 * kAttentionPartial * sizeof(float);
    return st;
}

huffllm_status huffllm_cache_attention(const huffllm_cache *cache, const huffllm_attention *args, void *workspace, size_t workspace_bytes,
                                       int32_t *err_flag, huffllm_stream stream) {
    clear_error();
    huffllm_status st = check_attention(cache, args, true);
    if (st != HUFFLLM_OK) return st;
    const huffllm_attention &a = *args;
    if (!a.q || !a.out || !workspace) return fail(HUFFLLM_ERR_INVALID_ARG, "null pointer");
    if (!aligned(a.q, 2) || !aligned(a.out, 2) || !aligned(workspace, 256) || !aligned(err_flag, 4))
        return fail(HUFFLLM_ERR_INVALID_ARG, "q and out must be 2-byte, workspace 256-byte, err_flag 4-byte aligned");
    size_t need = 0;
    if ((st = huffllm_attention_workspace_bytes(cache, args, &need)) != HUFFLLM_OK) return st;
    if (workspace_bytes < need) return fail(HUFFLLM_ERR_BUFFER_TOO_SMALL, "workspace too small");
    AttentionArgs k;
    memset(&k, 0, sizeof(k));
    k.c = cache_args(*cache);
    if (!stride_of(a.q_stride, (uint64_t)a.heads * cache->head_dim, &k.q_stride) || !stride_of(a.out_stride, (uint64_t)a.heads * cache->head_dim, &k.out_stride))
        return fail(HUFFLLM_ERR_INVALID_ARG, "stride below the values of a row (or above 2^40)");
    if (rows_overlap(a.q, a.out, (uint64_t)a.heads * cache->head_dim, k.q_stride, k.out_stride, a.rows)) return fail(HUFFLLM_ERR_INVALID_ARG, "out must not overlap q");
    k.q = a.q;
    k.out = a.out;
    k.starts = a.starts;
    k.rows = (uint32_t)a.rows;
    k.heads = a.heads;
    k.group = a.heads / cache->kv_heads;
    k.window = a.window;
    k.sinks = a.sinks;
    const uint64_t page_blocks = cache->page_tokens / kCacheBlock;
    k.page_recip = page_blocks == 1 ? 0xFFFFFFFFu : (uint32_t)((1ull << 32) / page_blocks);
    k.scale = a.scale;
    k.err = err_flag;
    k.tickets = (unsigned int *)workspace;
    k.partials = (float *)((uint8_t *)workspace + kAttentionCtas * sizeof(unsigned int));
    DeviceInfo dev;
    if ((st = device_info(&dev)) != HUFFLLM_OK) return st;
    return launched(launch_attention(k, dev.sms, (cudaStream_t)stream), "attention");
}

huffllm_status huffllm_sample(const huffllm_sampling *args, huffllm_stream stream) {
    clear_error();
    if (!args) return fail(HUFFLLM_ERR_INVALID_ARG, "null pointer");
    const huffllm_sampling &a = *args;
    if (!a.logits || !a.uniform || !a.tokens) return fail(HUFFLLM_ERR_INVALID_ARG, "null pointer");
    if (a.logits_type > HUFFLLM_ELEM_16 || a.dtype > HUFFLLM_FP16) return fail(HUFFLLM_ERR_INVALID_ARG, "unknown type");
    if (a.rows == 0 || a.vocab == 0) return fail(HUFFLLM_ERR_INVALID_ARG, "rows and vocab must be at least 1");
    if (a.rows > (1ull << 24) || a.vocab > kMost) return fail(HUFFLLM_ERR_UNSUPPORTED, "at most 2^24 rows and 2^31 - 1 tokens");
    if (!aligned(a.logits, a.logits_type == HUFFLLM_ELEM_16 ? 2 : 4)) return fail(HUFFLLM_ERR_INVALID_ARG, "pointers must be aligned to their types");
    for (const void *p : {(const void *)a.temperature, (const void *)a.top_k, (const void *)a.top_p, (const void *)a.min_p, (const void *)a.uniform, (const void *)a.tokens})
        if (!aligned(p, 4)) return fail(HUFFLLM_ERR_INVALID_ARG, "pointers must be aligned to their types");
    SamplingArgs s;
    memset(&s, 0, sizeof(s));
    if (!stride_of(a.stride, a.vocab, &s.stride)) return fail(HUFFLLM_ERR_INVALID_ARG, "stride below the vocabulary (or above 2^40)");
    s.logits = a.logits;
    s.temperature = a.temperature;
    s.top_k = a.top_k;
    s.top_p = a.top_p;
    s.min_p = a.min_p;
    s.uniform = a.uniform;
    s.tokens = a.tokens;
    s.rows = (uint32_t)a.rows;
    s.vocab = (uint32_t)a.vocab;
    s.type = a.logits_type == HUFFLLM_ELEM_F32 ? 0 : a.dtype == HUFFLLM_BF16 ? 1 : 2;
    DeviceInfo dev;
    const huffllm_status st = device_info(&dev);
    if (st != HUFFLLM_OK) return st;
    return launched(launch_sampling(s, dev.sms, (cudaStream_t)stream), "sampling");
}

}  // extern "C"
