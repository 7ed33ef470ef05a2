// Residual addition and root-mean-square norm between two products:
//     h = x + delta,  sum = h (rounded to x's type),  out = h / sqrt(mean(h^2) + eps) * gain (rounded to 16 bits)
// One CTA per vector and one pass: a thread keeps its values of h in registers while the squares' sum is taken, so x and delta are
// read once and sum and out written once.  (Vectors longer than the registers of a CTA hold are read twice, the second time from L2;
// every element is read by the thread that writes it, so sum may lie over x or delta either way.)  The sum of squares is taken in
// fp32 in a fixed order: eight at a time, a thread's, a warp's, the CTA's.
#include <cuda_runtime.h>
#include <type_traits>

#include "decode_common.cuh"
#include "epilogue.cuh"

namespace huffllm {

constexpr int kNormMaxThreads = 1024;
enum NormForm { kAligned, kPhased, kLoose };

// ITEMS groups of 8 values per thread, 0: as many as the vector has, in two passes.
// FORM says which columns a group is.  kAligned: eight that follow each other, every vector and group on 16-byte boundaries.  kPhased: eight that
// follow each other in memory from a multiple of eight values on; the vectors start anywhere, but all of them at the same place within
// eight values (packed vectors of an odd length do), `phase` values behind the first group's start, so that all but the outermost groups
// move in 16-byte pieces.  kLoose: eight that are blockDim.x columns apart, value by value.  (2048 x 5001 in 16 bits: phased 24 us, loose 41.)
// X16, DT: x in 16 bits; delta 0: none, 1: fp32, 2: 16 bits.  (Types that are asked about at run time make every load wait for the one
// before: 2048 x 8192 in 16 bits 45 us.)
template <bool F16, bool X16, int DT, int ITEMS, int FORM>
__global__ void __launch_bounds__(kNormMaxThreads) add_rms_norm_kernel(const __grid_constant__ NormArgs A) {
    __shared__ float s_sum[32];
    constexpr int N = ITEMS ? ITEMS : 1;
    const uint32_t tid = threadIdx.x, nt = blockDim.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t cols = (uint32_t)A.cols;                    // (at most 2^31)
    const uint64_t v = blockIdx.x;
    pdl_launch_dependents();
    const uint32_t phase = FORM == kPhased ? (uint32_t)(v * A.x_stride) & 7u : 0u;
    // (in front of the first column: wraps to more than `cols`)
    auto column = [&](uint32_t it, int j) -> uint32_t { return FORM == kLoose ? tid + (it * 8 + j) * nt : (tid + it * nt) * 8 + j - phase; };
    auto whole = [&](uint32_t it) -> bool { return column(it, 0) < cols && (FORM == kAligned || column(it, 7) < cols); };
    // Eight values as they lie in memory, and widened: all of a vector's loads are under way before the first value is looked at.
    auto load8 = [&](const void *p, uint64_t at, auto is16, uint32_t it, uint32_t (&r)[8]) {
        constexpr bool k16 = decltype(is16)::value;
#pragma unroll
        for (int j = 0; j < 8; ++j) r[j] = 0u;
        bool rest = FORM == kLoose;
        if (FORM != kLoose) {
            const bool in = whole(it);
            const uint4 zero = make_uint4(0, 0, 0, 0), *q = (const uint4 *)((const uint8_t *)p + ((int64_t)at + (int32_t)column(it, 0)) * (k16 ? 2 : 4));
            const uint4 a = in ? __ldcg(q) : zero;
            r[0] = a.x, r[1] = a.y, r[2] = a.z, r[3] = a.w;
            if (!k16) {
                const uint4 b = in ? __ldcg(q + 1) : zero;
                r[4] = b.x, r[5] = b.y, r[6] = b.z, r[7] = b.w;
            }
            rest = FORM == kPhased && !in;
        }
        if (rest) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool in = column(it, j) < cols;
                if (!k16) r[j] = in ? __ldcg((const unsigned int *)p + at + column(it, j)) : 0u;
                else if (FORM == kLoose) r[j] = in ? __ldcg((const unsigned short *)p + at + column(it, j)) : 0u;
                else if (in) r[j >> 1] |= (uint32_t)__ldcg((const unsigned short *)p + at + column(it, j)) << (16 * (j & 1));
            }
        }
    };
    auto widen8 = [](auto is16, const uint32_t (&r)[8], float (&o)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (!decltype(is16)::value) o[j] = __uint_as_float(r[j]);
            else if (FORM != kLoose) o[j] = widen16<F16>((uint16_t)(r[j >> 1] >> (16 * (j & 1))));
            else o[j] = widen16<F16>((uint16_t)r[j]);
        }
    };
    using Is16 = std::true_type;
    using XType = std::bool_constant<X16>;
    using DType = std::bool_constant<DT == 2>;
    auto store8 = [&](void *p, uint64_t at, bool is16, uint32_t it, const float (&o)[8]) {
        if (FORM != kLoose && whole(it)) {
            uint8_t *const q = (uint8_t *)p + ((int64_t)at + (int32_t)column(it, 0)) * (is16 ? 2 : 4);
            if (is16) {
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = round16<F16>(o[2 * j]) | (uint32_t)round16<F16>(o[2 * j + 1]) << 16;
                *(uint4 *)q = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
                ((float4 *)q)[0] = make_float4(o[0], o[1], o[2], o[3]);
                ((float4 *)q)[1] = make_float4(o[4], o[5], o[6], o[7]);
            }
        } else if (FORM != kAligned) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (column(it, j) < cols) store_value<F16>(p, at + column(it, j), is16, o[j]);
        }
    };
    // (the same for every vector, so from L1 where it cannot come in one piece)
    auto load_gain = [&](uint32_t it, uint32_t (&r)[8]) {
        if (!A.gain) return;
        if constexpr (FORM == kAligned) {
            load8(A.gain, 0, Is16{}, it, r);
        } else {
            if (FORM == kPhased && phase == 0 && whole(it)) {
                load8(A.gain, 0, Is16{}, it, r);
                return;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) r[j] = column(it, j) < cols ? __ldg(A.gain + column(it, j)) : 0u;
            if (FORM == kPhased) {
#pragma unroll
                for (int j = 0; j < 4; ++j) r[j] = r[2 * j] | r[2 * j + 1] << 16;
            }
        }
    };
    auto widen_gain = [&](const uint32_t (&r)[8], float (&o)[8]) {
        if (A.gain) {
            widen8(Is16{}, r, o);
            return;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = 1.0f;
    };
    auto load_h = [&](uint32_t it, uint32_t (&x)[8], uint32_t (&d)[8]) {
        load8(A.x, v * A.x_stride, XType{}, it, x);
        if (DT) load8(A.delta, v * A.delta_stride, DType{}, it, d);
    };
    auto widen_h = [&](const uint32_t (&x)[8], const uint32_t (&d)[8], float (&h)[8]) {
        widen8(XType{}, x, h);
        if (DT) {
            float f[8];
            widen8(DType{}, d, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) h[j] += f[j];
        }
    };
    auto squares = [](const float (&h)[8]) -> float {
        float s = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) s = fmaf(h[j], h[j], s);
        return s;
    };

    float h[N][8], gain[8], total = 0.0f;
    uint32_t g_raw[8], x_raw[N][8], d_raw[N][8];
    pdl_wait_prior_grid();                                        // (for everything that is read: gain may be as young as x)
    if (ITEMS == 1) load_gain(0, g_raw);
    const uint32_t groups = (cols + phase + 8 * nt - 1) / (8 * nt);       // of a thread
    if (ITEMS) {
#pragma unroll
        for (int it = 0; it < ITEMS; ++it) load_h(it, x_raw[it], d_raw[it]);
#pragma unroll
        for (int it = 0; it < ITEMS; ++it) {
            widen_h(x_raw[it], d_raw[it], h[it]);
            total += squares(h[it]);
        }
        if (A.sum) {
#pragma unroll
            for (int it = 0; it < ITEMS; ++it) store8(A.sum, v * A.sum_stride, X16, it, h[it]);
        }
    } else {
#pragma unroll 2
        for (uint32_t it = 0; it < groups; ++it) {
            load_h(it, x_raw[0], d_raw[0]);
            widen_h(x_raw[0], d_raw[0], h[0]);
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
    auto finish = [&](uint32_t it, float (&y)[8]) {
        widen_gain(g_raw, gain);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = y[j] * scale * gain[j];
        store8(A.out, v * A.out_stride, true, it, y);
    };
    if (ITEMS) {
#pragma unroll
        for (int it = 0; it < ITEMS; ++it) {
            if (ITEMS > 1) load_gain(it, g_raw);
            finish(it, h[it]);
        }
    } else {
        for (uint32_t it = 0; it < groups; ++it) {
            load_h(it, x_raw[0], d_raw[0]);
            load_gain(it, g_raw);
            widen_h(x_raw[0], d_raw[0], h[0]);
            if (A.sum) store8(A.sum, v * A.sum_stride, X16, it, h[0]);
            finish(it, h[0]);
        }
    }
}

template <bool F16, bool X16, int DT, int ITEMS, int FORM>
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
    return cudaLaunchKernelEx(&cfg, add_rms_norm_kernel<F16, X16, DT, ITEMS, FORM>, a);
}

template <bool F16, bool X16, int DT, int FORM>
static cudaError_t launch_norm_items(const NormArgs &a, uint32_t vectors, cudaStream_t stream) {
    const uint64_t groups = (a.cols + (FORM == kPhased ? 7 : 0) + 7) / 8;
    auto threads = [&](uint64_t items) -> uint32_t {
        const uint64_t t = ((groups + items - 1) / items + 31) / 32 * 32;
        return (uint32_t)(t < (uint64_t)kNormMaxThreads ? t : (uint64_t)kNormMaxThreads);
    };
    // One group of eight a thread where that makes a CTA of at most 1024 threads; where there are vectors for many rounds of CTAs anyway (eight a B200's SM), two or
    // four from 513 threads on, so that an SM's CTAs are more and wait for their sums at different times.  (us with one / two / four groups:
    // 296 x 8192 in 16 bits 5.3 / 6.0 / 6.3, 2048 x 8192 25.4 / 23.8 / 25.5; 2048 x 4096 in fp32 19.5 / 21.1 / 23.7; 4096 x 16384 - / 105 / 88.)
    const bool many = vectors >= 8 * 148;
    if (groups <= 512 || (groups <= 1024 && !many)) return launch_norm_one<F16, X16, DT, 1, FORM>(a, vectors, threads(1), stream);
    if (groups <= 1024 || (groups <= 2048 && !many)) return launch_norm_one<F16, X16, DT, 2, FORM>(a, vectors, threads(2), stream);
    if (groups <= 4096) return launch_norm_one<F16, X16, DT, 4, FORM>(a, vectors, threads(4), stream);
    return launch_norm_one<F16, X16, DT, 0, FORM>(a, vectors, kNormMaxThreads, stream);
}

template <bool F16, bool X16, int DT>
static cudaError_t launch_norm_form(const NormArgs &a, uint32_t vectors, cudaStream_t stream) {
    const uint64_t strides[4] = {a.x_stride, DT ? a.delta_stride : a.x_stride, a.sum ? a.sum_stride : a.x_stride, a.out_stride};
    const bool is16[4] = {X16, DT ? DT == 2 : X16, X16, true};
    bool own = true, same = true;
    for (int i = 0; i < 4; ++i) {
        own = own && strides[i] % (is16[i] ? 8 : 4) == 0;
        same = same && strides[i] % 8 == strides[0] % 8;
    }
    const bool based = !(((uintptr_t)a.x | (DT ? (uintptr_t)a.delta : 0) | (uintptr_t)a.sum | (uintptr_t)a.gain | (uintptr_t)a.out) & 15);
    if (based && own && a.cols % 8 == 0) return launch_norm_items<F16, X16, DT, kAligned>(a, vectors, stream);
    // (phased / loose, us, x in fp32 and delta in 16 bits: 64 x 1001 2.8 / 2.6, 64 x 5001 4.7 / 3.6, 148 x 5001 4.5 / 6.2, 600 x 1001 4.8 / 4.5, 1500 x 1001
    // 7.0 / 8.2, 1500 x 251 5.3 / 3.8, 1500 x 5001 22 / 33; 1 x 11001 4.4 / 6.8)
    if (based && same && (a.cols > 8192 || vectors * a.cols >= 640000)) return launch_norm_items<F16, X16, DT, kPhased>(a, vectors, stream);
    return launch_norm_items<F16, X16, DT, kLoose>(a, vectors, stream);
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
