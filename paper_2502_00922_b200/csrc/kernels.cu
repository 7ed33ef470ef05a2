// The register-path kernels of decode and of the products that hand out fp32 sums, the dense comparison product and small copies.
#include "huff_kernel.cuh"

namespace huffllm {

// ------------------------------------------------------------------------------ plain bf16 GEMV

// The dense product the compressed path competes with: y = W x for uncompressed bf16 matrices, written as a streaming
// kernel so that it is a fair opponent.  One launch takes a list of matrices (the same launch groups as the compressed
// path).  A warp takes one row at a time and walks it 4 KB per step: eight independent 16-byte loads per lane are in
// flight before the first is used (32 warps per SM: 128 KB per SM on its way, several times what the memory latency
// times an SM's share of the bandwidth asks for); x comes from L1; products in fp32, shuffle reduction.  Rows are dealt
// round-robin to the warps of the grid, so every SM keeps loads in flight until the launch ends.
__device__ __forceinline__ void fma_bf16x8(float &lo, float &hi, const uint4 &w, const uint4 &x) {
    const uint32_t wv[4] = {w.x, w.y, w.z, w.w}, xv[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        lo = fmaf(__uint_as_float(wv[j] << 16), __uint_as_float(xv[j] << 16), lo);
        hi = fmaf(__uint_as_float(wv[j] & 0xFFFF0000u), __uint_as_float(xv[j] & 0xFFFF0000u), hi);
    }
}

__global__ void __launch_bounds__(256, 4) plain_gemv_kernel(const __grid_constant__ PlainArgs A) {
    const uint32_t lane = threadIdx.x & 31;
    const uint32_t warp = (blockIdx.x * blockDim.x + threadIdx.x) >> 5, nwarps = (gridDim.x * blockDim.x) >> 5;
    // launched like the compressed path: the next launch may start early, and this one asks for its first weights before
    // the launch in front of it has finished; x is read only after that
    pdl_launch_dependents();
    bool waited_prior = false;
    uint32_t mi = 0;
    for (uint32_t u = warp; u < A.total_rows; u += nwarps) {
        while (mi + 1 < A.n_mats && u >= A.m[mi + 1].row_first) ++mi;
        const PlainMat &m = A.m[mi];
        const uint64_t r = u - m.row_first;
        const uint32_t nv = (uint32_t)(m.cols >> 3);                       // 16-byte pieces of a row
        const uint4 *wr = (const uint4 *)(m.w + r * m.cols), *xr = (const uint4 *)m.x;
        float a0 = 0.f, a1 = 0.f, b0 = 0.f, b1 = 0.f;
        for (uint32_t i = lane; i < nv; i += 256) {                        // eight pieces per lane and step
            uint4 p[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) p[j] = i + 32 * j < nv ? ldg_stream16(wr + i + 32 * j) : make_uint4(0, 0, 0, 0);
            if (!waited_prior) {
                pdl_wait_prior_grid();
                waited_prior = true;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint4 xv = i + 32 * j < nv ? __ldg(xr + i + 32 * j) : make_uint4(0, 0, 0, 0);
                if (j & 1) fma_bf16x8(b0, b1, p[j], xv);
                else fma_bf16x8(a0, a1, p[j], xv);
            }
        }
        float sum = (a0 + a1) + (b0 + b1);
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        if (lane == 0) m.y[r] = sum;
    }
}

// ------------------------------------------------------------------------------ small copies by a kernel

// Copies 16-byte pieces between device-accessible buffers (device memory, or pinned host memory that the device can
// address).  For the tens of kilobytes of activations and results of a decode step this is cheaper than a DMA copy:
// inside a CUDA graph a copy node between kernel nodes costs about 10 microseconds, this kernel about 3.
__global__ void __launch_bounds__(512) stage_copy_kernel(uint4 *__restrict__ dst, const uint4 *__restrict__ src, uint64_t n16) {
    pdl_launch_dependents();   // a product kernel behind this copy may do its set-up meanwhile: it waits for the copy before it reads x
    for (uint64_t i = (uint64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n16; i += (uint64_t)gridDim.x * blockDim.x) dst[i] = src[i];
}

cudaError_t launch_stage_copy(void *dst, const void *src, uint64_t bytes, uint32_t sms, cudaStream_t stream) {
    const uint64_t n16 = bytes / 16;
    uint64_t grid = (n16 + 511) / 512;
    if (grid > sms) grid = sms;
    if (grid == 0) return cudaSuccess;
    stage_copy_kernel<<<(uint32_t)grid, 512, 0, stream>>>((uint4 *)dst, (const uint4 *)src, n16);
    return cudaGetLastError();
}

// ------------------------------------------------------------------------------ launchers

// (Where rows go through shared memory is decided with the launch's shared memory: part_bytes.)
cudaError_t launch_decode(const KernelArgs &k, uint32_t grid, cudaStream_t stream) {
    return k.part_bytes ? launch_format<2, 1>(k, grid, stream) : launch_format<0, 1>(k, grid, stream);
}

cudaError_t launch_gemm(const KernelArgs &k, uint32_t grid, cudaStream_t stream) {
    if (k.batch == 1) return launch_format<1, 0>(k, grid, stream);           // one vector: multiply-adds on the FMA pipe
    if (k.batch > 8) return launch_slots<1, 8, 0, 2>(k, grid, stream);       // (the entry point sends only BF16 blobs of 8-bit tables here)
    return launch_format<1, 1>(k, grid, stream);
}

cudaError_t launch_plain_gemv(const PlainArgs &a, uint32_t sms, cudaStream_t stream) {
    const uint64_t blocks = ((uint64_t)a.total_rows + 7) / 8;               // 8 warps per CTA, a row per warp and turn
    const uint32_t grid = (uint32_t)(blocks < (uint64_t)sms * 4 ? blocks : (uint64_t)sms * 4);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(256);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, plain_gemv_kernel, a);
}

}  // namespace huffllm
