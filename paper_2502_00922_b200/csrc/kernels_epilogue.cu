// The register-path products with an epilogue.
#include "huff_kernel.cuh"

namespace huffllm {

cudaError_t launch_gemm(const EpiKernelArgs &k, uint32_t grid, cudaStream_t stream) {
    if (k.batch == 1) return launch_format<1, 0, 1>(k, grid, stream);
    if (k.batch > 8) return launch_slots<1, 8, 0, 2, 1>(k, grid, stream);
    return launch_format<1, 1, 1>(k, grid, stream);
}

}  // namespace huffllm
