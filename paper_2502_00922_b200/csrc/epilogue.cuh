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

// v / (1 + exp(-u)).  The fast exponential is off by |u| 2^-24 + 2^-22 of itself, the quotient by 2^-22.  For u = v far below zero, where the result is
// v exp(v), that is the result's relative error (1.7e-6 at -20, where half a unit in the last place of the sum alone, 2^-20, moves exp(v) by 1e-6); the
// exponential's share is below 1e-7 in absolute terms everywhere.  (expf costs four instructions more and shows in no 16-bit output.)
// (exp(-u) above 2^126: the quotient is 0 instead of a number below 1e-36.)
__device__ __forceinline__ float times_sigmoid(float v, float u) { return __fdividef(v, 1.0f + __expf(-u)); }

// v / 2 (1 + erf(v / sqrt 2)), from the tail q = erfc(z), z = |v| / sqrt 2:  v q / 2 below zero, v - v q / 2 above.
// erfc(z) = exp(-z^2) t P(t) with t = 1 / (1 + z / 2): P is the polynomial of degree 8 of least relative error on 0 <= z <= 12
// (Lawson's reweighted least squares), 1.5e-7 in fp32; the fast exponential adds v^2 2^-25 + 2^-22.  No cancellation where v is far below zero, where 1 + erf(v / sqrt 2) has it.
__device__ __forceinline__ float gelu(float v) {
    const float a = fabsf(v), t = __fdividef(1.0f, fmaf(0.353553390593274f, a, 1.0f));
    float p = -0.05936381220817566f;
    p = fmaf(p, t, 0.2860138416290283f);
    p = fmaf(p, t, -0.4901793599128723f);
    p = fmaf(p, t, 0.2814750075340271f);
    p = fmaf(p, t, -0.02897183783352375f);
    p = fmaf(p, t, 0.2036784291267395f);
    p = fmaf(p, t, 0.24285362660884857f);
    p = fmaf(p, t, 0.28240957856178284f);
    p = fmaf(p, t, 0.28208446502685547f);
    const float q = 0.5f * t * p * __expf(-0.5f * v * v);
    return v < 0.0f ? v * q : v - fminf(v, 64.0f) * q;          // (infinity: q is 0)
}

__device__ __forceinline__ float activated(float v, uint32_t act) {
    if (act == HUFFLLM_ACT_SILU) return times_sigmoid(v, v);
    if (act == HUFFLLM_ACT_RELU) return v < 0.0f ? 0.0f : v;                   // (a NaN stays one)
    // 1 + tanh(t) = 2 / (1 + exp(-2 t)): no cancellation here either; 2 sqrt(2 / pi)
    if (act == HUFFLLM_ACT_GELU_TANH) return times_sigmoid(v, 1.59576912160573f * v * fmaf(0.044715f * v, v, 1.0f));
    return gelu(v);
}
// `act` on N values, by calls: the activations' code stands in a kernel once, apart from what every launch runs.  (Inlined, and not
// even run: 22016 x 4096 at 12 vectors 47.4 us, without any such code 45.2; FP16 11008 x 4096 at 24 38.7 / 37.1.)
static __device__ __noinline__ float4 activate4(float4 v, uint32_t act) {
    return make_float4(activated(v.x, act), activated(v.y, act), activated(v.z, act), activated(v.w, act));
}
static __device__ __noinline__ float activate1(float v, uint32_t act) { return activated(v, act); }
template <int N>
__device__ __forceinline__ void activate(float (&v)[N], uint32_t act) {
    if (act == HUFFLLM_ACT_NONE) return;
    if constexpr (N < 4) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = activate1(v[i], act);
    } else {
        static_assert(N % 4 == 0, "fours");
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const float4 a = activate4(make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]), act);
            v[i] = a.x, v[i + 1] = a.y, v[i + 2] = a.z, v[i + 3] = a.w;
        }
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

// A lane's N sums of one row r = `row`: those of vectors n0, n0 + step, ...  The lanes of a warp hold rows that follow each other, from a
// multiple of 16 on (lane % 16 = row % 16), so that the other factor of a gated output is what lane ^ 8 holds.  ok: the row exists.

// Their residuals (zero where there are none), all loads under way together: asked about the type once per load, each waited for the one
// before (8192 x 28672 at 64 vectors 140 us, with neither residual nor activation 128).
template <bool F16, int N>
__device__ __forceinline__ void load_residuals(const EpiMat &e, float (&r)[N], uint32_t n0, uint32_t step, uint32_t batch, uint64_t row, bool ok) {
#pragma unroll
    for (int i = 0; i < N; ++i) r[i] = 0.0f;
    if (!e.residual || !ok) return;
    const uint64_t at = (uint64_t)n0 * e.residual_stride + row, more = (uint64_t)step * e.residual_stride;
    if (e.out16) {
        const unsigned short *p = (const unsigned short *)e.residual + at;
        unsigned short raw[N];
#pragma unroll
        for (int i = 0; i < N; ++i, p += more) raw[i] = n0 + step * i < batch ? __ldcg(p) : 0;
#pragma unroll
        for (int i = 0; i < N; ++i) r[i] = widen16<F16>(raw[i]);
    } else {
        const float *p = (const float *)e.residual + at;
#pragma unroll
        for (int i = 0; i < N; ++i, p += more)
            if (n0 + step * i < batch) r[i] = __ldcg(p);
    }
}
template <bool F16>
__device__ __forceinline__ float load_bias(const EpiMat &e, uint64_t row, bool ok) {
    return e.bias && ok ? widen16<F16>(__ldg(e.bias + row)) : 0.0f;
}
template <bool F16, int N>
__device__ __forceinline__ void store_outputs(const EpiMat &e, const float (&v)[N], uint32_t n0, uint32_t step, uint32_t batch, uint64_t col, bool ok) {
    if (!ok) return;
    const uint64_t at = (uint64_t)n0 * e.out_stride + col, more = (uint64_t)step * e.out_stride;
    if (e.out16) {
        uint16_t *p = (uint16_t *)e.out + at;
#pragma unroll
        for (int i = 0; i < N; ++i, p += more)
            if (n0 + step * i < batch) *p = round16<F16>(v[i]);
    } else {
        float *p = (float *)e.out + at;
#pragma unroll
        for (int i = 0; i < N; ++i, p += more)
            if (n0 + step * i < batch) *p = v[i];
    }
}
// From sums to outputs; called by the whole warp.  Gated, two vectors at a time: lanes with gate rows finish the even ones, lanes with up rows the
// odd ones, one exchange for two outputs.
template <bool F16, int N>
__device__ __forceinline__ void finish_gated(const EpiMat &e, const float (&sum)[N], float bias, uint32_t n0, uint32_t step, uint32_t batch, uint64_t row,
                                             bool ok, uint32_t lane) {
    constexpr int M = N > 1 ? N / 2 : 1;
    const bool up = lane & 8;
    float v[M], w[M];
#pragma unroll
    for (int j = 0; j < M; ++j) {
        const float even = sum[N > 1 ? 2 * j : 0] + bias, odd = N > 1 ? sum[N > 1 ? 2 * j + 1 : 0] + bias : 0.0f;
        const float got = __shfl_xor_sync(0xFFFFFFFFu, up ? even : odd, 8);
        v[j] = up ? got : even;
        w[j] = up ? odd : got;
    }
    activate<M>(v, e.act);
#pragma unroll
    for (int j = 0; j < M; ++j) v[j] *= w[j];
    const uint64_t col = (row >> 4) * 8 + (row & 7);
    store_outputs<F16, M>(e, v, n0 + (up ? step : 0), 2 * step, batch, col, ok && col < e.gated_rows && (N > 1 || !up));
}
template <bool F16, int N>
__device__ __forceinline__ void finish_plain(const EpiMat &e, const float (&sum)[N], float bias, const float (&residual)[N], uint32_t n0, uint32_t step,
                                             uint32_t batch, uint64_t row, bool ok) {
    float v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = sum[i] + bias;
    activate<N>(v, e.act);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += residual[i];
    store_outputs<F16, N>(e, v, n0, step, batch, row, ok);
}

}  // namespace huffllm
