// What the host side of the root-mean-square norm (sp24_rms_norm.cu) and its kernels (sp24_rms_norm_kernel.cuh) share.
#pragma once

#include "sp24_rows.cuh"

namespace sp24 {

struct NormParams {
  int64_t rows, K;
  const void *x, *residual, *weight;
  void *h, *y;
  float *scale, *rstd;
  int64_t ldx, ldr, ldh, ldy;
  float eps;
  int32_t weight_f32;
};

struct NormGradParams {
  int64_t rows, K;
  const void *dy, *h, *weight, *dh;
  const float* rstd;
  void* dx;
  float* partial;  // gridDim.x rows of K: each block's part of dweight, or null
  int64_t lddy, ldh, lddh, lddx;
  int32_t weight_f32;
};

// ---- in sp24_rms_norm_{f16,bf16,f32}.cu: each type in a source file of its own, so that they compile side by side ----------------
// WHOLE rows (and weight): see load_vector.
template <typename T>
sp24_status launch_rms_norm(sp24_dtype out_type, const NormParams& p, bool whole, cudaStream_t s);
// blocks: set to the number of blocks and of rows of partial sums, at most one to an SM.
template <typename T>
sp24_status launch_rms_norm_grad(const NormGradParams& p, bool whole, int64_t& blocks, cudaStream_t s);

}  // namespace sp24
