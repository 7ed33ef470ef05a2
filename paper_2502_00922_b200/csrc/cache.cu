// The 4-bit cache: new tokens written, tokens read back.
//
// A warp has the tokens that a call brings of one block (up to 16), of one head, of its keys or of its values.  A lane has eight channels of a
// token, which come and go as 16 bytes, four lanes have a group.  Eight codes are a word of the keys as it lies; of the values, a word has four
// tokens of two channels, so these change places in shared memory, four by four bytes.  Where rows are many, bound by instructions (18.6 million warp
// instructions for 17 million values, half of them around the values: groups, addresses, places), where they are few by four
// loads that follow each other: starts, length, page, row.  8294 rows of eight heads of 128 written 31 us, read back 24; 64 rows of one token 5 us each.
#include <cuda_runtime.h>

#include "cache_rows.cuh"
#include "decode_common.cuh"
#include "epilogue.cuh"

namespace huffllm {

constexpr uint32_t kCacheWarps = 8;                   // of a CTA at most

// The rows of a call that lie in one block.
struct BlockRows {
    uint32_t row, count;           // the first of them, and how many
    uint32_t r;                    // its place in the block
    int64_t block;                 // number of the block of head 0 among the pool's, or -1
    uint32_t head_step;            // from there to the next head's
};

// Calls f(BlockRows) for every block that begins among the CTA's `rows` rows; a warp at a time, all lanes alike.
template <typename F>
__device__ __forceinline__ void for_blocks(const CacheArgs &C, const CacheRows &R, uint32_t rows, F f) {
    constexpr uint32_t kFull = 0xFFFFFFFFu;
    const uint32_t lane = threadIdx.x % 32, row = blockIdx.x * rows + lane;
    if (blockIdx.x == 0 && blockIdx.y == 0) report_faults(C, R.starts, R.rows, R.err);
    BlockRows B{row, 0, 0, -1, C.page_tokens / kCacheBlock};
    const uint32_t b = sequences_of_rows(R.starts, C.sequences, blockIdx.x * rows, rows);
    if (lane < rows && row < R.rows) {
        const Sequence S = sequence_of(C, R.starts, R.rows, b);
        const uint32_t i = row - S.first_row;
        const int32_t at = S.tokens - (int32_t)S.rows + (int32_t)i;
        if (!S.bad && row >= S.first_row && i < S.rows && at >= 0 && (at % kCacheBlock == 0 || i == 0 || at == 0)) {
            B.r = at % kCacheBlock;
            B.count = min(kCacheBlock - B.r, S.rows - i);
            const int32_t page = __ldcg(C.table + (uint64_t)b * C.table_stride + at / C.page_tokens);
            if (page >= 0 && (uint32_t)page < C.pages) B.block = (int64_t)page * C.kv_heads * B.head_step + at % C.page_tokens / kCacheBlock;
            else if (R.err) *R.err = (int32_t)b + 1;
        }
    }
    for (uint32_t who = __ballot_sync(kFull, B.block >= 0); who; who &= who - 1) {
        const int l = __ffs(who) - 1;
        f(BlockRows{__shfl_sync(kFull, B.row, l), __shfl_sync(kFull, B.count, l), __shfl_sync(kFull, B.r, l), (int64_t)__shfl_sync(kFull, (long long)B.block, l), B.head_step});
    }
}

// A code in 64 bits (a call: few values need it).
static __device__ __noinline__ float exact_code(float v, float m, float s) { return (float)fmin(fmax(rint(((double)v - (double)m) / (double)s), 0.0), 15.0); }

// Four words, a byte of each into every word of the result: out[i] has byte i of in[0], in[1], in[2], in[3].
__device__ __forceinline__ void transpose_bytes(const uint32_t (&in)[4], uint32_t (&out)[4]) {
    const uint32_t a = prmt(in[0], in[1], 0x5140), b = prmt(in[2], in[3], 0x5140), c = prmt(in[0], in[1], 0x7362), d = prmt(in[2], in[3], 0x7362);
    out[0] = prmt(a, b, 0x5410), out[1] = prmt(a, b, 0x7632), out[2] = prmt(c, d, 0x5410), out[3] = prmt(c, d, 0x7632);
}
// Token i of the four in a word of values, t4's.
__device__ __forceinline__ uint32_t token_of(uint32_t t4, uint32_t i) { return 2 * t4 + (i >> 1) + (i & 1) * 8; }

// Words 4 half .. 4 half + 3 of value rows (g) and tile j of 16 channels, tokens t4's: items of a block are 2 * dim.  Neighbouring items are neighbours in
// memory: the words of a lane, then the lanes of a row.
template <uint32_t DIM>
struct ValueItem {
    uint32_t t4, j, half, word;                            // word: into the block's words, of row g = 4 half; the next g is 4 lanes on
    static constexpr uint32_t kItems = DIM / 16 * 8;
    __device__ __forceinline__ explicit ValueItem(uint32_t i) {
        t4 = i / 4 % 4;
        half = i / 16 % 2;
        j = i % 4 + i / 32 * 4;
    }
    __device__ __forceinline__ bool exists() const { return j < DIM / 16; }
    __device__ __forceinline__ uint32_t at(uint32_t g) const { return value_byte_at(DIM, 2 * t4, 16 * j + 4 * half + g); }   // bytes into the block
};

template <uint32_t DIM, bool F16>
__global__ void __launch_bounds__(kCacheWarps * 32, DIM <= 128 ? 4 : 3) cache_append_kernel(const __grid_constant__ CacheArgs C, const __grid_constant__ CacheRows R,
                                                                        const uint32_t rows) {
    constexpr uint32_t CHUNKS = DIM / 8, AT_ONCE = 2, G = cache_groups(DIM), kFull = 0xFFFFFFFFu;
    __shared__ uint32_t s_codes[kCacheWarps][kCacheBlock * DIM / 8];       // [token][16 channels][2]: a byte is two channels, eight apart
    pdl_launch_dependents();
    pdl_wait_prior_grid();
    const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, warps = blockDim.x / 32;
    const bool wide = !(((uintptr_t)R.k | (uintptr_t)R.v) & 15) && R.k_stride % 8 == 0 && R.v_stride % 8 == 0;
    for_blocks(C, R, rows, [&](const BlockRows &B) {
        for (uint32_t task = blockIdx.y * warps + warp; task < 2 * C.kv_heads; task += gridDim.y * warps) {
            const uint32_t head = task / 2;
            auto write = [&](auto side_) {
                constexpr uint32_t side = decltype(side_)::value;
                const uint16_t *const x = (side ? R.v : R.k) + head * DIM;
                const uint64_t stride = side ? R.v_stride : R.k_stride;
                uint8_t *const block = C.pool + (uint64_t)(B.block + (int64_t)head * B.head_step) * cache_block_bytes(DIM);
                // four pieces of 16 bytes (a lane's, of two tokens or more) on their way together; tokens that the call does not bring are passed over
#pragma unroll 1
                for (uint32_t k0 = B.r * CHUNKS / 32; k0 * 32 < (B.r + B.count) * CHUNKS; k0 += AT_ONCE) {
                    uint4 raw[AT_ONCE];
#pragma unroll
                    for (uint32_t k = 0; k < AT_ONCE; ++k) {
                        const uint32_t i = (k0 + k) * 32 + lane, token = i / CHUNKS, chunk = i % CHUNKS;
                        raw[k] = make_uint4(0, 0, 0, 0);
                        if (token - B.r >= B.count) continue;      // (wraps in front of the first)
                        const uint16_t *const from = x + (uint64_t)(B.row + token - B.r) * stride + chunk * 8;
                        if (wide) {
                            raw[k] = __ldcg((const uint4 *)from);
                        } else {
                            uint32_t e[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) e[j] = __ldcg((const unsigned short *)from + j);
                            raw[k] = make_uint4(e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16);
                        }
                    }
#pragma unroll
                    for (uint32_t k = 0; k < AT_ONCE; ++k) {
                        if ((k0 + k) * 32 >= (B.r + B.count) * CHUNKS) break;
                        const uint32_t i = (k0 + k) * 32 + lane, token = i / CHUNKS, chunk = i % CHUNKS, group = chunk / 4, t4 = chunk % 4;
                        const uint32_t w[4] = {raw[k].x, raw[k].y, raw[k].z, raw[k].w};
                        // smallest and largest of the group, two at a time; a NaN stays one
                        using Two = std::conditional_t<F16, __half2, __nv_bfloat162>;
                        auto two = [](const uint32_t &u) { return *(const Two *)&u; };
                        auto word = [](const Two &t) { return *(const uint32_t *)&t; };
                        uint32_t low2 = word(__hmin2_nan(__hmin2_nan(two(w[0]), two(w[1])), __hmin2_nan(two(w[2]), two(w[3]))));
                        uint32_t high2 = word(__hmax2_nan(__hmax2_nan(two(w[0]), two(w[1])), __hmax2_nan(two(w[2]), two(w[3]))));
#pragma unroll
                        for (int o = 1; o < 4; o <<= 1) {
                            const uint32_t l = __shfl_xor_sync(kFull, low2, o), h = __shfl_xor_sync(kFull, high2, o);
                            low2 = word(__hmin2_nan(two(low2), two(l)));
                            high2 = word(__hmax2_nan(two(high2), two(h)));
                        }
                        const uint32_t low_turned = prmt(low2, 0, 0x1032), high_turned = prmt(high2, 0, 0x1032);
                        const float low = widen16<F16>((uint16_t)word(__hmin2_nan(two(low2), two(low_turned))));
                        const float high = widen16<F16>((uint16_t)word(__hmax2_nan(two(high2), two(high_turned))));
                        // (high - low) / 15 as fp32 has it: the quotient by the reciprocal, and once more what that leaves over (Markstein's division)
                        const float span = high - low, first = span * (1.0f / 15.0f), span15 = fmaf(fmaf(-15.0f, first, span), 1.0f / 15.0f, first);
                        __half s = __float2half_rn(span15), m = __float2half_rn(low);
                        const bool sound = __half2float(s) < INFINITY && fabsf(__half2float(m)) < INFINITY;
                        if (!sound) s = __ushort_as_half(0x7FFFu), m = __ushort_as_half(0);
                        const float fs = __half2float(s), fm = __half2float(m), by = sound && fs != 0.0f ? __fdividef(1.0f, 15.0f * fs) : 0.0f;
                        // The code is (x - m) / s rounded.  In fp32 the quotient is off by less than 15 * 1.5 * 2^-22 = 5.4e-6 (difference and product 2^-24, division two
                        // last places): 64 bits decide within 1e-5 of a border alone.  (Taken as a part of 15, which cuts it off at both ends for nothing; 1.5 * 2^23 more is whole.)
                        float code[8], edge = 0.0f;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            const float v = widen16<F16>((uint16_t)(w[j >> 1] >> (j & 1) * 16)), q = __saturatef((v - fm) * by);
                            code[j] = fmaf(q, 15.0f, 12582912.0f) - 12582912.0f;
                            edge = fmaxf(edge, fabsf(fmaf(q, 15.0f, -code[j])));
                        }
                        if (edge > 0.49999f && by != 0.0f) {
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                const float v = widen16<F16>((uint16_t)(w[j >> 1] >> (j & 1) * 16)), q = __saturatef((v - fm) * by);
                                if (fabsf(fmaf(q, 15.0f, -code[j])) > 0.49999f) code[j] = exact_code(v, fm, fs);
                            }
                        }
                        // (whole numbers in fp32: 2^23 more has them in its low bits)
                        auto join2 = [](float a, float b, float by) { return __float_as_uint(fmaf(b, by, a + 8388608.0f)); };
                        const bool here = token - B.r < B.count;
                        if (side == 0) {
                            const uint32_t even = __float_as_uint(fmaf(fmaf(fmaf(code[6], 16.0f, code[4]), 16.0f, code[2]), 16.0f, code[0] + 8388608.0f));
                            const uint32_t odd = __float_as_uint(fmaf(fmaf(fmaf(code[7], 16.0f, code[5]), 16.0f, code[3]), 16.0f, code[1] + 8388608.0f));
                            if (here) *(uint32_t *)(block + key_word_at(DIM, token, group, t4)) = prmt(even, odd, 0x5410);
                        } else {
                            // eight channels of 16 come from this lane, the others from its neighbour; each gets half of their bytes
                            const uint32_t front = prmt(join2(code[0], code[1], 256.0f), join2(code[2], code[3], 256.0f), 0x5410);
                            const uint32_t back = prmt(join2(code[4], code[5], 256.0f), join2(code[6], code[7], 256.0f), 0x5410);
                            const uint32_t other = __shfl_xor_sync(kFull, lane & 1 ? front : back, 1);
                            if (here) s_codes[warp][token * (DIM / 8) + chunk] = lane & 1 ? other | back << 4 : front | other << 4;
                        }
                        if (here && t4 == 0) {
                            *(__half *)(block + (side ? value_scale_at(DIM, token, group) : key_scale_at(DIM, token, group))) = s;
                            *(__half *)(block + (side ? value_offset_at(DIM, token, group) : key_offset_at(DIM, token, group))) = m;
                            // (keys' offsets are read in pairs, and what is read is multiplied by 0: it must be a number)
                            if (G % 2 && side == 0 && group + 1 == G) *(__half *)(block + key_offset_at(DIM, token, group + 1)) = __ushort_as_half(0);
                        }
                    }
                }
                if (side == 0) return;
                __syncwarp();
#pragma unroll
                for (uint32_t i = 0; i < (ValueItem<DIM>::kItems + 31) / 32 * 32; i += 32) {
                    const ValueItem<DIM> item(i + lane);
                    if (!item.exists()) continue;
                    uint32_t in[4], out[4], mask = 0;
#pragma unroll
                    for (uint32_t j = 0; j < 4; ++j) {
                        const uint32_t token = token_of(item.t4, j);
                        in[j] = s_codes[warp][token * (DIM / 8) + item.j * 2 + item.half];
                        mask |= token - B.r < B.count ? 1u << j : 0u;
                    }
                    if (mask == 0) continue;
                    transpose_bytes(in, out);
#pragma unroll
                    for (uint32_t g = 0; g < 4; ++g) {
                        uint8_t *const to = block + item.at(g);
                        if (mask == 15u) {
                            *(uint32_t *)to = out[g];
                        } else {
#pragma unroll
                            for (uint32_t j = 0; j < 4; ++j)
                                if (mask >> j & 1) to[j] = (uint8_t)(out[g] >> 8 * j);
                        }
                    }
                }
                __syncwarp();
            };
            if (task % 2) write(std::integral_constant<uint32_t, 1>());
            else write(std::integral_constant<uint32_t, 0>());
        }
    });
}

template <uint32_t DIM, bool F16>
__global__ void __launch_bounds__(kCacheWarps * 32, DIM <= 128 ? 5 : 3) cache_read_kernel(const __grid_constant__ CacheArgs C, const __grid_constant__ CacheRows R,
                                                                      const uint32_t rows) {
    constexpr uint32_t CHUNKS = DIM / 8, EACH = kCacheBlock * CHUNKS / 32;
    __shared__ uint32_t s_codes[kCacheWarps][kCacheBlock * DIM / 8];
    pdl_launch_dependents();
    pdl_wait_prior_grid();
    const uint32_t lane = threadIdx.x % 32, warp = threadIdx.x / 32, warps = blockDim.x / 32;
    const bool wide = !(((uintptr_t)R.k | (uintptr_t)R.v) & 15) && R.k_stride % 8 == 0 && R.v_stride % 8 == 0;
    for_blocks(C, R, rows, [&](const BlockRows &B) {
        for (uint32_t task = blockIdx.y * warps + warp; task < 2 * C.kv_heads; task += gridDim.y * warps) {
            const uint32_t head = task / 2;
            auto read = [&](auto side_) {
                constexpr uint32_t side = decltype(side_)::value;
                uint16_t *const base = side ? R.v : R.k;
                if (!base) return;
                const uint64_t stride = side ? R.v_stride : R.k_stride;
                const uint8_t *const block = C.pool + (uint64_t)(B.block + (int64_t)head * B.head_step) * cache_block_bytes(DIM);
                if (side) {
#pragma unroll
                    for (uint32_t i = 0; i < (ValueItem<DIM>::kItems + 31) / 32 * 32; i += 32) {
                        const ValueItem<DIM> item(i + lane);
                        if (!item.exists()) continue;
                        uint32_t in[4], out[4];
#pragma unroll
                        for (uint32_t g = 0; g < 4; ++g) in[g] = __ldcg((const uint32_t *)(block + item.at(g)));
                        transpose_bytes(in, out);
#pragma unroll
                        for (uint32_t j = 0; j < 4; ++j) s_codes[warp][token_of(item.t4, j) * (DIM / 8) + item.j * 2 + item.half] = out[j];
                    }
                    __syncwarp();
                }
#pragma unroll
                for (uint32_t k = 0; k < EACH; ++k) {
                    const uint32_t i = k * 32 + lane, token = i / CHUNKS, chunk = i % CHUNKS, group = chunk / 4, t4 = chunk % 4;
                    if (token - B.r >= B.count) continue;
                    const float s = __half2float(__ushort_as_half(__ldcg((const unsigned short *)(block + (side ? value_scale_at(DIM, token, group) : key_scale_at(DIM, token, group))))));
                    const float m = __half2float(__ushort_as_half(__ldcg((const unsigned short *)(block + (side ? value_offset_at(DIM, token, group) : key_offset_at(DIM, token, group))))));
                    // (the code in the low four bits: behind 2^23, as conversions go through a slower pipe)
                    auto number = [](uint32_t u) { return __uint_as_float((u & 15u) | 0x4B000000u) - 8388608.0f; };
                    float v[8];
                    if (side) {
                        const uint32_t pair = token * (DIM / 8) + chunk / 2 * 2, shift = chunk % 2 * 4;
                        const uint32_t c0 = s_codes[warp][pair] >> shift, c1 = s_codes[warp][pair + 1] >> shift;
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[j] = fmaf(s, number(c0 >> 8 * j), m), v[4 + j] = fmaf(s, number(c1 >> 8 * j), m);
                    } else {
                        const uint32_t word = __ldcg((const uint32_t *)(block + key_word_at(DIM, token, group, t4)));
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] = fmaf(s, number(word >> ((j & 1) * 16 + (j >> 1) * 4)), m);
                    }
                    const uint64_t to = (uint64_t)(B.row + token - B.r) * stride + head * DIM + chunk * 8;
                    if (R.f32) {
                        float *const o = (float *)base + to;
                        if (wide) {
                            ((float4 *)o)[0] = make_float4(v[0], v[1], v[2], v[3]);
                            ((float4 *)o)[1] = make_float4(v[4], v[5], v[6], v[7]);
                        } else {
#pragma unroll
                            for (int j = 0; j < 8; ++j) o[j] = v[j];
                        }
                    } else {
                        uint32_t w[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) w[j] = round16x2<F16>(v[2 * j], v[2 * j + 1]);
                        if (wide) {
                            *(uint4 *)(base + to) = make_uint4(w[0], w[1], w[2], w[3]);
                        } else {
#pragma unroll
                            for (int j = 0; j < 8; ++j) base[to + j] = (uint16_t)(w[j >> 1] >> (j & 1) * 16);
                        }
                    }
                }
                if (side) __syncwarp();
            };
            if (task % 2) read(std::integral_constant<uint32_t, 1>());
            else read(std::integral_constant<uint32_t, 0>());
        }
    });
}

template <uint32_t DIM>
static cudaError_t launch_move(bool append, const CacheArgs &c, const CacheRows &r, cudaStream_t stream) {
    // A warp for every head and side, up to eight a CTA.  Sixteen rows a CTA, as many as a block has, where sequences bring some eight rows or more
    // (48 sequences with 34 rows each, eight heads: 106 us with a CTA a row); else one.
    const uint32_t tasks = 2 * c.kv_heads, warps = tasks < kCacheWarps ? tasks : kCacheWarps;
    const uint32_t rows = r.rows / 8 >= c.sequences ? kCacheBlock : 1;
    const dim3 grid((r.rows + rows - 1) / rows, (tasks + warps - 1) / warps);
    auto kernel = append ? (c.fp16 ? cache_append_kernel<DIM, true> : cache_append_kernel<DIM, false>) : (c.fp16 ? cache_read_kernel<DIM, true> : cache_read_kernel<DIM, false>);
    return launch_behind(kernel, grid, warps * 32, 0, stream, c, r, rows);
}
static cudaError_t launch_dim(bool append, const CacheArgs &c, const CacheRows &r, cudaStream_t stream) {
    switch (c.dim) {
        case 64: return launch_move<64>(append, c, r, stream);
        case 96: return launch_move<96>(append, c, r, stream);
        case 128: return launch_move<128>(append, c, r, stream);
        case 192: return launch_move<192>(append, c, r, stream);
        default: return launch_move<256>(append, c, r, stream);
    }
}
cudaError_t launch_cache_append(const CacheArgs &c, const CacheRows &r, cudaStream_t stream) { return launch_dim(true, c, r, stream); }
cudaError_t launch_cache_read(const CacheArgs &c, const CacheRows &r, cudaStream_t stream) { return launch_dim(false, c, r, stream); }

}  // namespace huffllm
