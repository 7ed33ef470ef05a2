// The tensor-core products with an epilogue.
#include "tc_kernel.cuh"

namespace huffllm {

cudaError_t launch_gemm_tc(const EpiTcArgs &t, uint32_t grid, cudaStream_t stream) { return launch_tc_format<1>(t, grid, stream); }

}  // namespace huffllm
