// The GEMM kernels over the problems of many experts for INT8 operands.
#include "sp24_expert_kernel.cuh"

namespace sp24 {
template <int KIND>
sp24_status launch_experts(int group, TileShape t, bool sparse, const sp24_gemm_desc* d, const GemmParams& p, const void* A, const void* meta, const void* B,
                           cudaStream_t s) {
  return launch_group_shape<KIND>(group, t, sparse, d, p, A, meta, B, s);
}
template sp24_status launch_experts<1>(int, TileShape, bool, const sp24_gemm_desc*, const GemmParams&, const void*, const void*, const void*, cudaStream_t);
}  // namespace sp24
