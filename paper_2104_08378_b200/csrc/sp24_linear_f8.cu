// The GEMM kernels with the epilogue of sp24_linear for 8-bit floating-point operands.
#include "sp24_gemm_kernel.cuh"

namespace sp24 {
template <int KIND>
sp24_status launch_linear(TileShape t, bool sparse, bool b_mn, const sp24_gemm_desc* d, const GemmParams& p, const void* A,
                          const void* meta, const void* B, cudaStream_t s) {
  return launch_shape<KIND, true>(t, sparse, b_mn, d, p, A, meta, B, s);
}
template sp24_status launch_linear<3>(TileShape, bool, bool, const sp24_gemm_desc*, const GemmParams&, const void*, const void*,
                                     const void*, cudaStream_t);
}  // namespace sp24
