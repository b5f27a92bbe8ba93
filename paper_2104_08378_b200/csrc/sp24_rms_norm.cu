// Root-mean-square norm with the residual's addition and 8-bit results, and its gradient: argument checks, entry points, the sums of partial rows.
#include "sp24_rms_norm.cuh"

namespace sp24 {
namespace {

// out[k] = the sum of `parts` rows, in their order within each of eight shares and then the shares in theirs.
__global__ void __launch_bounds__(256) column_sums_kernel(const float* partial, int64_t parts, int64_t K, float* out) {
  __shared__ float share[8][33];
  wait_for_stream();
  const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
  const int64_t k = (int64_t)blockIdx.x * 32 + lane;
  float sum = 0.f;
  if (k < K)
    for (int64_t b = group; b < parts; b += 8) sum += partial[b * K + k];
  share[group][lane] = sum;
  __syncthreads();
  if (group == 0 && k < K) {
    for (int i = 1; i < 8; ++i) sum += share[i][lane];
    out[k] = sum;
  }
}

// Blocks of the gradient's kernel at most, one to an SM: each keeps a row of dweight's sums in the workspace.  (Where no device tells its SMs, room for the largest.)
int64_t most_grad_blocks(int64_t rows) {
  const int64_t sms = sm_count() > 1 ? sm_count() : 592;
  return rows < sms ? rows : sms;
}

}  // namespace

sp24_status column_sums(const float* partial, int64_t parts, int64_t K, float* out, cudaStream_t s) {
  return launch_overlapped(column_sums_kernel, dim3((unsigned)((K + 31) / 32)), dim3(256), 0, s, 1, partial, parts, K, out);
}

}  // namespace sp24

using namespace sp24;

extern "C" sp24_status sp24_rms_norm(sp24_dtype t, int64_t rows, int64_t K, const void* x, int64_t ldx, const void* residual,
                                     int64_t ldr, const void* weight, sp24_dtype weight_type, float eps, void* h, int64_t ldh,
                                     sp24_dtype out_type, void* y, int64_t ldy, float* scale, float* rstd, void* stream) {
  SP24_RETURN_IF(!is_float_type(t) || (out_type != t && !is_code_type(out_type)), SP24_ERR_DTYPE);
  SP24_RETURN_IF(weight && weight_type != t && weight_type != SP24_F32, SP24_ERR_DTYPE);
  SP24_RETURN_IF(rows < 0 || K < 1 || K > kMostColumns, SP24_ERR_SHAPE);
  SP24_RETURN_IF(!(eps >= 0.f) || (h && !residual) || (h && h == y), SP24_ERR_UNSUPPORTED);
  if (rows == 0) return SP24_OK;
  SP24_RETURN_IF(!x || !y || (is_code_type(out_type) && !scale), SP24_ERR_NULL);
  SP24_RETURN_IF(!row_fits(rows, K, ldx) || (residual && !row_fits(rows, K, ldr)) || (h && !row_fits(rows, K, ldh)) || !row_fits(rows, K, ldy), SP24_ERR_STRIDE);
  const size_t es = elem_bytes(t), os = elem_bytes(out_type);
  SP24_RETURN_IF(!aligned(x, es) || !aligned(residual, es) || !aligned(h, es) || !aligned(y, os) || !aligned(weight, elem_bytes(weight_type)) ||
                     !aligned(scale, 4) || !aligned(rstd, 4),
                 SP24_ERR_ALIGN);
  sp24_status st = check_arch();
  if (st != SP24_OK) return st;
  const NormParams p = {rows, K, x, residual, weight, h, y, scale, rstd, ldx, ldr, ldh, ldy, eps, weight_type == SP24_F32};
  const bool whole = K * es % 16 == 0 && whole_rows(x, rows, ldx, es, 16) && whole_rows(residual, rows, ldr, es, 16) && whole_rows(h, rows, ldh, es, 16) &&
                     whole_rows(y, rows, ldy, os, 16 / es * os) && aligned16(weight);
  return with_float_type(t, [&](auto type) { return launch_rms_norm<typename decltype(type)::type>(out_type, p, whole, static_cast<cudaStream_t>(stream)); });
}

extern "C" size_t sp24_rms_norm_backward_workspace_bytes(int64_t rows, int64_t K) {
  if (rows <= 0 || K < 1 || K > kMostColumns) return 0;
  return (size_t)most_grad_blocks(rows) * (size_t)K * sizeof(float);
}

extern "C" sp24_status sp24_rms_norm_backward(sp24_dtype t, int64_t rows, int64_t K, const void* dy, int64_t lddy, const void* h,
                                              int64_t ldh, const void* weight, sp24_dtype weight_type, const float* rstd,
                                              const void* dh, int64_t lddh, void* dx, int64_t lddx, float* dweight, void* workspace,
                                              size_t workspace_bytes, void* stream) {
  SP24_RETURN_IF(!is_float_type(t) || (weight && weight_type != t && weight_type != SP24_F32), SP24_ERR_DTYPE);
  SP24_RETURN_IF(rows < 0 || K < 1 || K > kMostColumns, SP24_ERR_SHAPE);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (rows == 0) {
    if (!dweight) return SP24_OK;
    SP24_RETURN_IF(!aligned(dweight, 4), SP24_ERR_ALIGN);
    const sp24_status st = check_arch();
    return st != SP24_OK ? st : cuda_status(cudaMemsetAsync(dweight, 0, (size_t)K * sizeof(float), s));
  }
  SP24_RETURN_IF(!dy || !h || !rstd || !dx, SP24_ERR_NULL);
  SP24_RETURN_IF(!row_fits(rows, K, lddy) || !row_fits(rows, K, ldh) || (dh && !row_fits(rows, K, lddh)) || !row_fits(rows, K, lddx), SP24_ERR_STRIDE);
  const size_t es = elem_bytes(t);
  SP24_RETURN_IF(!aligned(dy, es) || !aligned(h, es) || !aligned(dh, es) || !aligned(dx, es) || !aligned(weight, elem_bytes(weight_type)) ||
                     !aligned(rstd, 4) || !aligned(dweight, 4),
                 SP24_ERR_ALIGN);
  SP24_RETURN_IF(dweight && (!workspace || !aligned16(workspace) || workspace_bytes < sp24_rms_norm_backward_workspace_bytes(rows, K)),
                 SP24_ERR_WORKSPACE);
  sp24_status st = check_arch();
  if (st != SP24_OK) return st;
  int64_t blocks = 0;
  const NormGradParams p = {rows, K, dy, h, weight, dh, rstd, dx, dweight ? static_cast<float*>(workspace) : nullptr, lddy, ldh, lddh, lddx, weight_type == SP24_F32};
  const bool whole = K * es % 16 == 0 && whole_rows(dy, rows, lddy, es, 16) && whole_rows(h, rows, ldh, es, 16) && whole_rows(dh, rows, lddh, es, 16) &&
                     whole_rows(dx, rows, lddx, es, 16) && aligned16(weight);
  st = with_float_type(t, [&](auto type) { return launch_rms_norm_grad<typename decltype(type)::type>(p, whole, blocks, s); });
  if (st != SP24_OK || !dweight) return st;
  return column_sums(static_cast<const float*>(workspace), blocks, K, dweight, s);
}
