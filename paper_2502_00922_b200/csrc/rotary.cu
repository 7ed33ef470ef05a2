// Rotary positions with several axes: pair i of a head turns by positions[axis(i)][token] * frequencies[i].
#include <cuda_runtime.h>

#include "decode_common.cuh"
#include "decode_step.h"
#include "epilogue.cuh"

namespace huffllm {

__device__ __forceinline__ uint32_t axis_of(const RotaryArgs &A, uint32_t i) { return A.axis_bits[i / 16] >> i % 16 * 2 & 3u; }

// Sine and cosine of position * frequency.  The product has 55 bits and is taken in turns: as the sum of two numbers of 64 bits each, product and
// 1 / (2 pi) both (Dekker's product, its rest by fused multiplication), so that what is left behind the whole turns is right to fp32 for every
// position and every frequency up to 2^40 and more.  (In one number 2^31 turns are off by 2^-21 of one, 2^48 by a tenth.)
__device__ __forceinline__ float2 turn_of(int32_t position, float frequency) {
    constexpr double kTurn = 0.15915494309189533577, kTurnRest = -9.839338337591243e-18;      // 1 / (2 pi), and what the first leaves of it
    const double p = position, f = frequency, product = p * f, product_rest = fma(p, f, -product);
    const double turns = product * kTurn, rest = fma(product, kTurn, -turns) + fma(product, kTurnRest, product_rest * kTurn);
    const double left = (turns - rint(turns)) + rest;
    float s, c;
    sincospif((float)(2.0 * (left - rint(left))), &s, &c);
    return make_float2(c, s);
}

template <bool F16>
__global__ void __launch_bounds__(128) rotary_kernel(const __grid_constant__ RotaryArgs A) {
    pdl_launch_dependents();
    pdl_wait_prior_grid();
    const uint32_t token = blockIdx.x, pairs = A.rot / 2;
    for (uint32_t i = threadIdx.x; i < (A.dim - A.rot) + pairs; i += blockDim.x) {
        const bool turned = i < pairs;
        const float2 cs = turned ? turn_of(__ldcg(A.positions + (uint64_t)axis_of(A, i) * A.tokens + token), __ldcg(A.frequencies + i)) : make_float2(1, 0);
        const uint32_t a = !turned ? A.rot + i - pairs : A.neighbours ? 2 * i : i, b = !turned ? a : A.neighbours ? 2 * i + 1 : i + pairs;
        for (int w = 0; w < 2; ++w) {
            const uint16_t *in = A.in[w] + token * A.in_stride[w];
            uint16_t *out = A.out[w] + token * A.out_stride[w];
            for (uint32_t h = 0; h < A.heads[w]; ++h) {
                const uint16_t xa = __ldcg(in + h * A.dim + a), xb = __ldcg(in + h * A.dim + b);
                if (!turned) {
                    out[h * A.dim + a] = xa;
                    continue;
                }
                const float va = widen16<F16>(xa), vb = widen16<F16>(xb);
                out[h * A.dim + a] = round16<F16>(va * cs.x - vb * cs.y);
                out[h * A.dim + b] = round16<F16>(vb * cs.x + va * cs.y);
            }
        }
    }
}

// Heads whose channels lie on 16-byte boundaries: a thread turns eight channels with the eight half a rotary_dim away (or four pairs of
// neighbours), in as many heads as threads leave it.  A CTA has a token; its sines and cosines meet in shared memory while the
// heads are on their way.  5003 tokens of 32 heads of 128: 14.7 us, 5.6 TB/s, 0.85 of the measured copy rate (value by value 44 us); what is left is the way
// of a CTA from positions by sines to its heads.  One token 7.1 us, most of them the call.
constexpr uint32_t kRotaryThreads = 256, kRotaryEach = 2;
template <bool F16, bool NEIGHBOURS>
__global__ void __launch_bounds__(kRotaryThreads) rotary_wide_kernel(const __grid_constant__ RotaryArgs A) {
    __shared__ float4 s_turn[256];                       // cosines and sines of two pairs; of an item's pairs `turned` apart, so that neighbours read neighbours
    pdl_launch_dependents();
    pdl_wait_prior_grid();
    const uint32_t token = blockIdx.x, pairs = A.rot / 2, tid = threadIdx.x;
    const uint32_t turned = NEIGHBOURS ? A.rot / 8 : A.rot / 16;          // items of a head: turned ones, and pieces that are copied
    const uint32_t items = turned + (A.dim - A.rot) / 8, all = items * (A.heads[0] + A.heads[1]);
    const uint32_t step = blockDim.x * kRotaryEach;
    bool known = false;
    for (uint32_t base = 0; base < all; base += step) {
        uint4 x[kRotaryEach], y[kRotaryEach];
        const uint16_t *from[kRotaryEach];
        uint16_t *to[kRotaryEach];
        uint32_t part[kRotaryEach];
#pragma unroll
        for (uint32_t k = 0; k < kRotaryEach; ++k) {
            const uint32_t i = base + k * blockDim.x + tid, h = i / items;
            part[k] = i % items;
            const uint32_t which = h < A.heads[0] ? 0 : 1, head = which ? h - A.heads[0] : h;
            const uint32_t at = head * A.dim + (part[k] < turned ? part[k] * 8 : A.rot + (part[k] - turned) * 8);
            from[k] = A.in[which] + token * A.in_stride[which] + at;
            to[k] = A.out[which] + token * A.out_stride[which] + at;
            if (i >= all) {
                to[k] = nullptr;
                continue;
            }
            x[k] = __ldcg((const uint4 *)from[k]);
            if (!NEIGHBOURS && part[k] < turned) y[k] = __ldcg((const uint4 *)(from[k] + pairs));
        }
        if (!known) {
            constexpr uint32_t PER = NEIGHBOURS ? 4 : 8;              // pairs of an item
            for (uint32_t i = tid; i < pairs; i += blockDim.x)
                ((float2 *)s_turn)[(i % PER / 2 * turned + i / PER) * 2 + i % 2] =
                    turn_of(__ldcg(A.positions + (uint64_t)axis_of(A, i) * A.tokens + token), __ldcg(A.frequencies + i));
            __syncthreads();
            known = true;
        }
#pragma unroll
        for (uint32_t k = 0; k < kRotaryEach; ++k) {
            if (!to[k]) continue;
            if (part[k] >= turned) {
                if (to[k] != from[k]) *(uint4 *)to[k] = x[k];
                continue;
            }
            const uint32_t a[4] = {x[k].x, x[k].y, x[k].z, x[k].w}, b[4] = {y[k].x, y[k].y, y[k].z, y[k].w};
            uint32_t c[4], d[4];
            auto lo = [](uint32_t w) { return widen16<F16>((uint16_t)w); };
            auto hi = [](uint32_t w) { return widen16<F16>((uint16_t)(w >> 16)); };
            auto both = [](float l, float h) { return round16x2<F16>(l, h); };
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) {
                if constexpr (NEIGHBOURS) {
                    const float4 t = s_turn[j / 2 * turned + part[k]];
                    const float cosine = j % 2 ? t.z : t.x, sine = j % 2 ? t.w : t.y;
                    c[j] = both(lo(a[j]) * cosine - hi(a[j]) * sine, hi(a[j]) * cosine + lo(a[j]) * sine);
                } else {
                    const float4 t = s_turn[j * turned + part[k]];
                    c[j] = both(lo(a[j]) * t.x - lo(b[j]) * t.y, hi(a[j]) * t.z - hi(b[j]) * t.w);
                    d[j] = both(lo(b[j]) * t.x + lo(a[j]) * t.y, hi(b[j]) * t.z + hi(a[j]) * t.w);
                }
            }
            *(uint4 *)to[k] = make_uint4(c[0], c[1], c[2], c[3]);
            if (!NEIGHBOURS) *(uint4 *)(to[k] + pairs) = make_uint4(d[0], d[1], d[2], d[3]);
        }
    }
}

cudaError_t launch_rotary(const RotaryArgs &a, cudaStream_t stream) {
    bool wide = a.dim % 8 == 0 && a.rot % (a.neighbours ? 8 : 16) == 0;
    for (int w = 0; w < 2; ++w)
        if (a.heads[w]) wide = wide && !(((uintptr_t)a.in[w] | (uintptr_t)a.out[w]) & 15) && a.in_stride[w] % 8 == 0 && a.out_stride[w] % 8 == 0;
    if (!wide) return launch_behind(a.fp16 ? rotary_kernel<true> : rotary_kernel<false>, dim3(a.tokens), 128, 0, stream, a);
    const uint32_t items = ((a.neighbours ? a.rot / 8 : a.rot / 16) + (a.dim - a.rot) / 8) * (a.heads[0] + a.heads[1]);
    // (as few threads as go through a token's items in whole rounds)
    const uint32_t rounds = (items + kRotaryThreads * kRotaryEach - 1) / (kRotaryThreads * kRotaryEach), each = rounds * kRotaryEach;
    const uint32_t threads = ((items + each - 1) / each + 31) / 32 * 32;
    auto kernel = a.neighbours ? (a.fp16 ? rotary_wide_kernel<true, true> : rotary_wide_kernel<false, true>)
                               : (a.fp16 ? rotary_wide_kernel<true, false> : rotary_wide_kernel<false, false>);
    return launch_behind(kernel, dim3(a.tokens), threads, 0, stream, a);
}

}  // namespace huffllm
