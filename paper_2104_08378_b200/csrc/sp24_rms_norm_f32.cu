// The root-mean-square norm and its gradient on FP32 rows.
#include "sp24_rms_norm_kernel.cuh"

namespace sp24 {
template sp24_status launch_rms_norm<float>(sp24_dtype, const NormParams&, bool, cudaStream_t);
template sp24_status launch_rms_norm_grad<float>(const NormGradParams&, bool, int64_t&, cudaStream_t);
}  // namespace sp24
