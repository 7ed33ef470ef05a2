// The tensor-core products that hand out fp32 sums.
#include "tc_kernel.cuh"

namespace huffllm {

cudaError_t launch_gemm_tc(const TcArgs &t, uint32_t grid, cudaStream_t stream) {
    return t.k.fmt ? launch_tc_fp16<0>(t, grid, stream) : launch_tc_bf16<0>(t, grid, stream);
}

}  // namespace huffllm
