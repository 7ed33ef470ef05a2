// The tensor-core products of BF16 blobs with an epilogue.
#include "tc_kernel.cuh"

namespace huffllm {

cudaError_t launch_gemm_tc(const EpiTcArgs &t, uint32_t grid, cudaStream_t stream) {
    return t.k.fmt ? launch_gemm_tc_fp16(t, grid, stream) : launch_tc_bf16<1>(t, grid, stream);
}

}  // namespace huffllm
