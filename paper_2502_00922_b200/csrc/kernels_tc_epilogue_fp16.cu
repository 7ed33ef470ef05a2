// The tensor-core products of FP16 blobs with an epilogue.
#include "tc_kernel.cuh"

namespace huffllm {

cudaError_t launch_gemm_tc_fp16(const EpiTcArgs &t, uint32_t grid, cudaStream_t stream) { return launch_tc_fp16<1>(t, grid, stream); }

}  // namespace huffllm
