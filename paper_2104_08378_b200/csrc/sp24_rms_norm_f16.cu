// The root-mean-square norm and its gradient on FP16 rows.
#include "sp24_rms_norm_kernel.cuh"

namespace sp24 {
template sp24_status launch_rms_norm<__half>(sp24_dtype, const NormParams&, bool, cudaStream_t);
template sp24_status launch_rms_norm_grad<__half>(const NormGradParams&, bool, int64_t&, cudaStream_t);
}  // namespace sp24
