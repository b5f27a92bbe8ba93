// Root-mean-square norm with the residual's addition and 8-bit results, and its gradient.
#include "sp24_rows.cuh"

namespace sp24 {
namespace {

struct NormParams {
  int64_t rows, K;
  const void *x, *residual, *weight;
  void *h, *y;
  float *scale, *rstd;
  int64_t ldx, ldr, ldh, ldy;
  float eps;
  int32_t weight_f32;
};

// Rows of any length and alignment: a block to a row, two passes over it (the second from the caches).  The scale of an 8-bit row needs no
// pass of its own: max |n| = rstd max |h w|.
template <typename T, typename OUT>
__global__ void __launch_bounds__(1024) rms_norm_kernel(const NormParams p) {
  __shared__ RowSums sums;
  int turn = 0;
  wait_for_stream();
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    const T* r = p.residual ? static_cast<const T*>(p.residual) + row * p.ldr : nullptr;
    T* h = p.h ? static_cast<T*>(p.h) + row * p.ldh : nullptr;
    OUT* y = static_cast<OUT*>(p.y) + row * p.ldy;
    auto weight = [&](int64_t k) { return p.weight ? load_weight<T>(p.weight, p.weight_f32, k) : 1.f; };
    auto value = [&](int64_t k) { return r ? to_float(round_to<T>(to_float(x[k]) + to_float(r[k]))) : to_float(x[k]); };
    float sum = 0.f;
    uint32_t top = 0;
    for (int64_t k = threadIdx.x; k < p.K; k += blockDim.x) {
      const float v = value(k);
      sum = fmaf(v, v, sum);
      if (is_code<OUT>) top = max(top, magnitude(v * weight(k)));
    }
    sums.reduce(sum, top, turn);
    const float rstd = rsqrtf(sum / (float)p.K + p.eps);
    if (threadIdx.x == 0 && p.rstd) p.rstd[row] = rstd;
    float inv = 0.f;
    if (is_code<OUT>) {
      const float scale = row_scale<OUT>(__uint_as_float(top), rstd, &inv);
      if (threadIdx.x == 0) p.scale[row] = scale;
    }
    for (int64_t k = threadIdx.x; k < p.K; k += blockDim.x) {
      const float v = value(k);
      if (h) h[k] = round_to<T>(v);
      if constexpr (is_code<OUT>) y[k] = to_code<OUT>(v * weight(k) * inv);
      else y[k] = round_to<OUT>(v * rstd * weight(k));
    }
  }
}

struct NormGradParams {
  int64_t rows, K;
  const void *dy, *h, *weight, *dh;
  const float* rstd;
  void* dx;
  float* partial;  // gridDim.x rows of K: each block's part of dweight, or null
  int64_t lddy, ldh, lddh, lddx;
  int32_t weight_f32;
};

template <typename T>
__global__ void __launch_bounds__(1024) rms_norm_grad_kernel(const NormGradParams p) {
  __shared__ RowSums sums;
  int turn = 0;
  wait_for_stream();
  bool first = true;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, first = false) {
    const T* dy = static_cast<const T*>(p.dy) + row * p.lddy;
    const T* h = static_cast<const T*>(p.h) + row * p.ldh;
    const T* dh = p.dh ? static_cast<const T*>(p.dh) + row * p.lddh : nullptr;
    T* dx = static_cast<T*>(p.dx) + row * p.lddx;
    auto weight = [&](int64_t k) { return p.weight ? load_weight<T>(p.weight, p.weight_f32, k) : 1.f; };
    const float rstd = p.rstd[row];
    float sum = 0.f;
    uint32_t unused = 0;
    for (int64_t k = threadIdx.x; k < p.K; k += blockDim.x) sum = fmaf(to_float(dy[k]) * weight(k), to_float(h[k]), sum);
    sums.reduce(sum, unused, turn);
    const float along = sum / (float)p.K * rstd * rstd;
    float* part = p.partial ? p.partial + blockIdx.x * p.K : nullptr;
    for (int64_t k = threadIdx.x; k < p.K; k += blockDim.x) {
      const float g = to_float(dy[k]), v = to_float(h[k]);
      float d = rstd * fmaf(-v, along, g * weight(k));
      if (dh) d += to_float(dh[k]);
      dx[k] = round_to<T>(d);
      if (part) part[k] = fmaf(g * v, rstd, first ? 0.f : part[k]);
    }
  }
}

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

// Blocks of the gradient's kernel: each keeps a row of dweight's sums in the workspace.
constexpr int64_t kMostPartials = 592;
int64_t grad_blocks(int64_t rows) { return rows < kMostPartials ? rows : kMostPartials; }

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
  SP24_RETURN_IF(!(eps >= 0.f) || (h && !residual), SP24_ERR_UNSUPPORTED);
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
  return with_float_type(t, [&](auto type) {
    using T = typename decltype(type)::type;
    return with_out_type<T>(out_type, [&](auto out) {
      using OUT = typename decltype(out)::type;
      return launch_overlapped(rms_norm_kernel<T, OUT>, dim3((unsigned)(rows < 65535 ? rows : 65535)), dim3(row_threads(K)), 0,
                               static_cast<cudaStream_t>(stream), 1, p);
    });
  });
}

extern "C" size_t sp24_rms_norm_backward_workspace_bytes(int64_t rows, int64_t K) {
  if (rows <= 0 || K < 1 || K > kMostColumns) return 0;
  return (size_t)grad_blocks(rows) * (size_t)K * sizeof(float);
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
  const int64_t blocks = grad_blocks(rows);
  const NormGradParams p = {rows, K, dy, h, weight, dh, rstd, dx, dweight ? static_cast<float*>(workspace) : nullptr, lddy, ldh, lddh, lddx, weight_type == SP24_F32};
  st = with_float_type(t, [&](auto type) {
    using T = typename decltype(type)::type;
    return launch_overlapped(rms_norm_grad_kernel<T>, dim3((unsigned)blocks), dim3(row_threads(K)), 0, s, 1, p);
  });
  if (st != SP24_OK || !dweight) return st;
  return column_sums(static_cast<const float*>(workspace), blocks, K, dweight, s);
}
