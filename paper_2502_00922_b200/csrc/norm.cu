// Residual addition and root-mean-square norm between two products:
//     h = x + delta,  sum = h (rounded to x's type),  out = h / sqrt(mean(h^2) + eps) * gain (rounded to 16 bits)
// One CTA per vector and one pass: a thread keeps its values of h in registers while the squares' sum is taken, so x and delta are
// read once and sum and out written once.  (Vectors longer than the registers of a CTA hold are read twice, the second time from L2;
// every element is read by the thread that writes it, so sum may lie over x or delta either way.)  The sum of squares is taken in
// fp32 in a fixed order: eight at a time, a thread's, a warp's, the CTA's.
// `gain` does not come from the kernel in front and is asked for before the wait for it.
#include <cuda_runtime.h>
#include <cstdlib>

#include "decode_common.cuh"
#include "epilogue.cuh"

namespace huffllm {

constexpr int kNormMaxThreads = 1024;

// ITEMS groups of 8 values per thread, 0: as many as the vector has, in two passes.  VEC: everything is 16-byte aligned and a group is
// eight columns that follow each other; otherwise a group's values are blockDim.x columns apart.
// X16, DT: x in 16 bits; delta 0: none, 1: fp32, 2: 16 bits.  (Types that are asked about at run time make every load wait for the one
// before: 2048 x 8192 in 16 bits 45 us.)
template <bool F16, bool X16, int DT, int ITEMS, bool VEC>
__global__ void __launch_bounds__(kNormMaxThreads) add_rms_norm_kernel(const __grid_constant__ NormArgs A) {
    __shared__ float s_sum[32];
    constexpr int N = ITEMS ? ITEMS : 1;
    const uint32_t tid = threadIdx.x, nt = blockDim.x, lane = tid & 31, warp = tid >> 5;
    const uint64_t cols = A.cols, v = blockIdx.x;
    pdl_launch_dependents();
    auto column = [&](uint64_t it, int j) -> uint64_t { return VEC ? (tid + it * nt) * 8 + j : tid + (it * 8 + j) * nt; };
    auto load8 = [&](const void *p, uint64_t at, bool is16, uint64_t it, float (&o)[8]) {
        if (VEC) {
            if (column(it, 0) >= cols) {
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = 0.0f;
                return;
            }
            if (is16) {
                const uint4 q = __ldcg((const uint4 *)((const uint16_t *)p + at + column(it, 0)));
                const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j] = widen16<F16>((uint16_t)(w[j >> 1] >> (16 * (j & 1))));
            } else {
                const float4 *q = (const float4 *)((const float *)p + at + column(it, 0));
                const float4 a = __ldcg(q), b = __ldcg(q + 1);
                o[0] = a.x, o[1] = a.y, o[2] = a.z, o[3] = a.w, o[4] = b.x, o[5] = b.y, o[6] = b.z, o[7] = b.w;
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = column(it, j) < cols ? load_value<F16>(p, at + column(it, j), is16) : 0.0f;
        }
    };
    auto store8 = [&](void *p, uint64_t at, bool is16, uint64_t it, const float (&o)[8]) {
        if (VEC) {
            if (column(it, 0) >= cols) return;
            if (is16) {
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = round16<F16>(o[2 * j]) | (uint32_t)round16<F16>(o[2 * j + 1]) << 16;
                *(uint4 *)((uint16_t *)p + at + column(it, 0)) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
                float4 *q = (float4 *)((float *)p + at + column(it, 0));
                q[0] = make_float4(o[0], o[1], o[2], o[3]);
                q[1] = make_float4(o[4], o[5], o[6], o[7]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (column(it, j) < cols) store_value<F16>(p, at + column(it, j), is16, o[j]);
        }
    };
    auto load_gain = [&](uint64_t it, float (&o)[8]) {
        if (!A.gain) {
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = 1.0f;
        } else {
            load8(A.gain, 0, true, it, o);
        }
    };
    auto load_h = [&](uint64_t it, float (&h)[8]) {
        load8(A.x, v * A.x_stride, X16, it, h);
        if (DT) {
            float d[8];
            load8(A.delta, v * A.delta_stride, DT == 2, it, d);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] += d[j];
        }
    };
    auto squares = [](const float (&h)[8]) -> float {
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) s = fmaf(h[j], h[j], s);
        return s;
    };

    float h[N][8], gain[1][8], total = 0.0f;
    if (ITEMS == 1) load_gain(0, gain[0]);
    pdl_wait_prior_grid();
    const uint64_t groups = (cols + 8 * nt - 1) / (8 * nt);       // of a thread
    if (ITEMS) {
#pragma unroll
        for (int it = 0; it < ITEMS; ++it) load_h(it, h[it]);
#pragma unroll
        for (int it = 0; it < ITEMS; ++it) total += squares(h[it]);
        if (A.sum) {
#pragma unroll
            for (int it = 0; it < ITEMS; ++it) store8(A.sum, v * A.sum_stride, X16, it, h[it]);
        }
    } else {
        for (uint64_t it = 0; it < groups; ++it) {
            load_h(it, h[0]);
            total += squares(h[0]);
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, o);
    if (lane == 0) s_sum[warp] = total;
    __syncthreads();
    total = lane < (nt >> 5) ? s_sum[lane] : 0.0f;
#pragma unroll
    for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, o);
    const float scale = rsqrtf(total / (float)cols + A.eps);
    if (ITEMS) {
#pragma unroll
        for (int it = 0; it < ITEMS; ++it) {
            if (ITEMS > 1) load_gain(it, gain[0]);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[it][j] = h[it][j] * scale * gain[0][j];
            store8(A.out, v * A.out_stride, true, it, h[it]);
        }
    } else {
        for (uint64_t it = 0; it < groups; ++it) {
            load_h(it, h[0]);
            if (A.sum) store8(A.sum, v * A.sum_stride, X16, it, h[0]);
            load_gain(it, gain[0]);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[0][j] = h[0][j] * scale * gain[0][j];
            store8(A.out, v * A.out_stride, true, it, h[0]);
        }
    }
}

template <bool F16, bool X16, int DT, int ITEMS, bool VEC>
static cudaError_t launch_norm_one(const NormArgs &a, uint32_t grid, uint32_t threads, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, add_rms_norm_kernel<F16, X16, DT, ITEMS, VEC>, a);
}

template <bool F16, bool X16, int DT, bool VEC>
static cudaError_t launch_norm_items(const NormArgs &a, uint32_t vectors, cudaStream_t stream) {
    const uint64_t groups = (a.cols + 7) / 8;
    auto threads = [&](uint64_t items) -> uint32_t {
        const uint64_t t = ((groups + items - 1) / items + 31) / 32 * 32;
        return (uint32_t)(t < (uint64_t)kNormMaxThreads ? t : (uint64_t)kNormMaxThreads);
    };
    int n = getenv("NITEMS") ? atoi(getenv("NITEMS")) : 0;
    if (n == 2) return launch_norm_one<F16, X16, DT, 2, VEC>(a, vectors, threads(2), stream);
    if (n == 4) return launch_norm_one<F16, X16, DT, 4, VEC>(a, vectors, threads(4), stream);
    if (groups <= (uint64_t)kNormMaxThreads) return launch_norm_one<F16, X16, DT, 1, VEC>(a, vectors, threads(1), stream);
    if (groups <= 2ull * kNormMaxThreads) return launch_norm_one<F16, X16, DT, 2, VEC>(a, vectors, threads(2), stream);
    return launch_norm_one<F16, X16, DT, 0, VEC>(a, vectors, kNormMaxThreads, stream);
}

template <bool F16, bool X16, int DT>
static cudaError_t launch_norm_form(const NormArgs &a, uint32_t vectors, cudaStream_t stream) {
    auto vec = [](const void *p, uint64_t stride, bool is16) { return !((uintptr_t)p & 15) && stride % (is16 ? 8 : 4) == 0; };
    const bool aligned = a.cols % 8 == 0 && vec(a.x, a.x_stride, X16) && (!DT || vec(a.delta, a.delta_stride, DT == 2)) &&
                         (!a.sum || vec(a.sum, a.sum_stride, X16)) && vec(a.gain, 0, true) && vec(a.out, a.out_stride, true);
    return aligned ? launch_norm_items<F16, X16, DT, true>(a, vectors, stream) : launch_norm_items<F16, X16, DT, false>(a, vectors, stream);
}

template <bool F16>
static cudaError_t launch_norm_types(const NormArgs &a, uint32_t vectors, cudaStream_t stream) {
    const int dt = !a.delta ? 0 : a.delta16 ? 2 : 1;
    if (a.x16)
        return dt == 0 ? launch_norm_form<F16, true, 0>(a, vectors, stream) : dt == 1 ? launch_norm_form<F16, true, 1>(a, vectors, stream)
                                                                                       : launch_norm_form<F16, true, 2>(a, vectors, stream);
    return dt == 0 ? launch_norm_form<F16, false, 0>(a, vectors, stream) : dt == 1 ? launch_norm_form<F16, false, 1>(a, vectors, stream)
                                                                                    : launch_norm_form<F16, false, 2>(a, vectors, stream);
}

cudaError_t launch_add_rms_norm(const NormArgs &a, uint32_t vectors, bool fp16, cudaStream_t stream) {
    return fp16 ? launch_norm_types<true>(a, vectors, stream) : launch_norm_types<false>(a, vectors, stream);
}

}  // namespace huffllm
