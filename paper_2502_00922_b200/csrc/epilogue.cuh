// What becomes of a product's sums before they leave the chip: bias, activation, gate times up, residual, rounding.
//
//   plain   out[b][r] = act(sum[b][r] + bias[r]) + residual[b][r]
//   gated   out[b][i] = act(sum[b][gate i] + bias[gate i]) * (sum[b][up i] + bias[up i])
//
// All in fp32, rounded once where out is 16 bits wide.  The matrix of a gated product has eight gate rows and the eight up rows
// of the same outputs in each group of 16 (huffllm_stack_gate_up): the warp that has a row group's sums, or the lanes l and l ^ 8 of
// one that reads an accumulator, hold both factors, and nothing has to meet across warps or CTAs for them.
// The warp that closes a row group does this: a handful of instructions per output, against the thousands that its weights took.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "huffllm.h"
#include "kernels.h"

namespace huffllm {

// v / (1 + exp(-u)).  (exp(-u) above 2^126: the quotient is 0 instead of a number below 1e-36.)
__device__ __forceinline__ float times_sigmoid(float v, float u) { return __fdividef(v, 1.0f + expf(-u)); }

// `act` on N values.  1 + tanh(t) = 2 / (1 + exp(-2 t)) and 1 + erf(t) = erfc(-t): no cancellation where v is far below zero.
template <int N>
__device__ __forceinline__ void activate(float (&v)[N], uint32_t act) {
    if (act == HUFFLLM_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = times_sigmoid(v[i], v[i]);
    } else if (act == HUFFLLM_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = v[i] < 0.0f ? 0.0f : v[i];          // (a NaN stays one)
    } else if (act == HUFFLLM_ACT_GELU_TANH) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = times_sigmoid(v[i], 1.59576912160573f * v[i] * fmaf(0.044715f * v[i], v[i], 1.0f));   // 2 sqrt(2 / pi)
    } else if (act == HUFFLLM_ACT_GELU) {
        // (one copy of a long function in code that runs cold: the values take their turns from local memory)
        float t[N];
#pragma unroll
        for (int i = 0; i < N; ++i) t[i] = v[i];
#pragma unroll 1
        for (int i = 0; i < N; ++i) t[i] = 0.5f * t[i] * erfcf(-0.707106781186548f * t[i]);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = t[i];
    }
}

template <bool F16>
__device__ __forceinline__ float widen16(uint16_t v) {
    return F16 ? __half2float(__ushort_as_half(v)) : __uint_as_float((uint32_t)v << 16);
}
template <bool F16>
__device__ __forceinline__ uint16_t round16(float v) {
    return F16 ? __half_as_ushort(__float2half_rn(v)) : __bfloat16_as_ushort(__float2bfloat16_rn(v));
}
// A value of the residual, past L1: the kernel in front may have written it, and may have read its place before.
template <bool F16>
__device__ __forceinline__ float load_value(const void *p, uint64_t at, bool is16) {
    return is16 ? widen16<F16>(__ldcg((const unsigned short *)p + at)) : __ldcg((const float *)p + at);
}
template <bool F16>
__device__ __forceinline__ void store_value(void *p, uint64_t at, bool is16, float v) {
    if (is16) ((uint16_t *)p)[at] = round16<F16>(v);
    else ((float *)p)[at] = v;
}

// The outputs of row group rg: tile[16 b + r] is the sum of vector b and the group's row r.  U outputs of a lane at a time, so that
// their residuals are under way together.
template <bool F16, int U>
__device__ __forceinline__ void finish_tile(const EpiMat &e, const float *tile, uint32_t batch, uint32_t rg, uint64_t rows, uint32_t lane) {
    const bool gated = e.gated_rows != 0, is16 = e.out16 != 0;
    const uint32_t shift = gated ? 3 : 4, per = 1u << shift, n = per * batch;
    const uint64_t first = (uint64_t)rg * per, end = gated ? e.gated_rows : rows;
#pragma unroll 1
    for (uint32_t o0 = lane; o0 < n; o0 += 32 * U) {
        float v[U], w[U];                                    // w: the second factor, or the residual
        bool ok[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t o = o0 + 32 * u, i = o & (per - 1), b = o >> shift;
            ok[u] = o < n && first + i < end;
            v[u] = w[u] = 0.0f;
            if (!ok[u]) continue;
            v[u] = tile[16 * b + i];
            if (e.bias) v[u] += widen16<F16>(__ldg(e.bias + (uint64_t)rg * 16 + i));
            if (gated) {
                w[u] = tile[16 * b + 8 + i];
                if (e.bias) w[u] += widen16<F16>(__ldg(e.bias + (uint64_t)rg * 16 + 8 + i));
            } else if (e.residual) {
                w[u] = load_value<F16>(e.residual, (uint64_t)b * e.residual_stride + first + i, is16);
            }
        }
        activate<U>(v, e.act);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t o = o0 + 32 * u;
            if (ok[u]) store_value<F16>(e.out, (uint64_t)(o >> shift) * e.out_stride + first + (o & (per - 1)), is16, gated ? v[u] * w[u] : v[u] + w[u]);
        }
    }
}

// The outputs of an accumulator's row `row` (of lane `lane`; the warp's 32 lanes hold rows that follow each other, from a multiple
// of 16 on) for vectors n0 .. n0 + CW - 1.  Called by the whole warp.
template <bool F16, int CW>
__device__ __forceinline__ void finish_columns(const EpiMat &e, const float (&sum)[CW], uint32_t n0, uint32_t batch, uint64_t row, bool row_ok,
                                               uint32_t lane) {
    const bool is16 = e.out16 != 0;
    const float bias = e.bias && row_ok ? widen16<F16>(__ldg(e.bias + row)) : 0.0f;
    if (e.gated_rows) {
        // lanes with gate rows finish the even vectors, lanes with up rows the odd ones: one exchange for two outputs
        const bool up = lane & 8;
        float v[CW / 2], w[CW / 2];
#pragma unroll
        for (int j = 0; j < CW / 2; ++j) {
            const float even = sum[2 * j] + bias, odd = sum[2 * j + 1] + bias;
            const float got = __shfl_xor_sync(0xFFFFFFFFu, up ? even : odd, 8);
            v[j] = up ? got : even;
            w[j] = up ? odd : got;
        }
        activate<CW / 2>(v, e.act);
        const uint64_t i = (row >> 4) * 8 + (row & 7);
        n0 += up ? 1 : 0;
#pragma unroll
        for (int j = 0; j < CW / 2; ++j)
            if (row_ok && n0 + 2 * j < batch && i < e.gated_rows) store_value<F16>(e.out, (uint64_t)(n0 + 2 * j) * e.out_stride + i, is16, v[j] * w[j]);
        return;
    }
    float v[CW];
#pragma unroll
    for (int i = 0; i < CW; ++i) v[i] = sum[i] + bias;
    activate<CW>(v, e.act);
    constexpr int U = CW < 8 ? CW : 8;
#pragma unroll
    for (int i0 = 0; i0 < CW; i0 += U) {
        if (e.residual) {
            float r[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                r[u] = row_ok && n0 + i0 + u < batch ? load_value<F16>(e.residual, (uint64_t)(n0 + i0 + u) * e.residual_stride + row, is16) : 0.0f;
#pragma unroll
            for (int u = 0; u < U; ++u) v[i0 + u] += r[u];
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (row_ok && n0 + i0 + u < batch) store_value<F16>(e.out, (uint64_t)(n0 + i0 + u) * e.out_stride + row, is16, v[i0 + u]);
    }
}

}  // namespace huffllm
