// Gated activation with 8-bit results, act(g) * u, and its gradient.
#include "sp24_act.cuh"
#include "sp24_rows.cuh"

namespace sp24 {
namespace {

struct GatedParams {
  int64_t rows, F;
  const void *g, *u;  // u: null for act(g) alone
  void* y;
  float* scale;
  int64_t ldg, ldu, ldy;
};

// Rows of any length and alignment: a block to a row; for 8-bit results a pass before it for the row's maximum.
template <typename T, typename OUT, int ACT>
__global__ void __launch_bounds__(1024) gated_act_kernel(const GatedParams p) {
  __shared__ RowSums sums;
  int turn = 0;
  wait_for_stream();
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const T* g = static_cast<const T*>(p.g) + row * p.ldg;
    const T* u = p.u ? static_cast<const T*>(p.u) + row * p.ldu : nullptr;
    OUT* y = static_cast<OUT*>(p.y) + row * p.ldy;
    auto value = [&](int64_t k) { return act_value<ACT>(to_float(g[k])) * (u ? to_float(u[k]) : 1.f); };
    float inv = 0.f;
    if (is_code<OUT>) {
      float top = 0.f, unused = 0.f;
      for (int64_t k = threadIdx.x; k < p.F; k += blockDim.x) top = max_abs(top, value(k), 0.f);
      sums.reduce(unused, top, turn);
      const float scale = row_scale<OUT>(finite_or_nan(top), 1.f, &inv);
      if (threadIdx.x == 0) p.scale[row] = scale;
    }
    for (int64_t k = threadIdx.x; k < p.F; k += blockDim.x) {
      if constexpr (is_code<OUT>) y[k] = to_code<OUT>(value(k) * inv);
      else y[k] = round_to<OUT>(value(k));
    }
  }
}

struct GatedGradParams {
  int64_t rows, F;
  const void *dy, *g, *u;
  void *dg, *du;
  int64_t lddy, ldg, ldu, lddg, lddu;
};

template <typename T, int ACT>
__global__ void __launch_bounds__(256) gated_act_grad_kernel(const GatedGradParams p) {
  wait_for_stream();
  for (int64_t row = blockIdx.y; row < p.rows; row += gridDim.y) {
    const T* dy = static_cast<const T*>(p.dy) + row * p.lddy;
    const T* g = static_cast<const T*>(p.g) + row * p.ldg;
    for (int64_t k = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; k < p.F; k += (int64_t)gridDim.x * blockDim.x) {
      float slope, d = to_float(dy[k]);
      const float value = act_and_slope<ACT>(to_float(g[k]), &slope);
      const float w = p.u ? to_float(static_cast<const T*>(p.u)[row * p.ldu + k]) : 1.f;
      static_cast<T*>(p.dg)[row * p.lddg + k] = round_to<T>(d * w * slope);
      if (p.du) static_cast<T*>(p.du)[row * p.lddu + k] = round_to<T>(d * value);
    }
  }
}

}  // namespace
}  // namespace sp24

using namespace sp24;

extern "C" sp24_status sp24_gated_act(sp24_dtype t, sp24_act act, int64_t rows, int64_t F, const void* g, int64_t ldg, const void* u,
                                      int64_t ldu, sp24_dtype out_type, void* y, int64_t ldy, float* scale, void* stream) {
  SP24_RETURN_IF(!is_float_type(t) || (out_type != t && !is_code_type(out_type)), SP24_ERR_DTYPE);
  SP24_RETURN_IF(!is_act(act), SP24_ERR_UNSUPPORTED);
  SP24_RETURN_IF(rows < 0 || F < 1 || F > kMostColumns, SP24_ERR_SHAPE);
  if (rows == 0) return SP24_OK;
  SP24_RETURN_IF(!g || !y || (is_code_type(out_type) && !scale), SP24_ERR_NULL);
  SP24_RETURN_IF(!row_fits(rows, F, ldg) || (u && !row_fits(rows, F, ldu)) || !row_fits(rows, F, ldy), SP24_ERR_STRIDE);
  const size_t es = elem_bytes(t);
  SP24_RETURN_IF(!aligned(g, es) || !aligned(u, es) || !aligned(y, elem_bytes(out_type)) || !aligned(scale, 4), SP24_ERR_ALIGN);
  const sp24_status st = check_arch();
  if (st != SP24_OK) return st;
  const GatedParams p = {rows, F, g, u, y, scale, ldg, ldu, ldy};
  return with_float_type(t, [&](auto type) {
    using T = typename decltype(type)::type;
    return with_out_type<T>(out_type, [&](auto out) {
      using OUT = typename decltype(out)::type;
      return with_act(act, [&](auto a) {
        return launch_overlapped(gated_act_kernel<T, OUT, decltype(a)::value>, dim3((unsigned)(rows < 65535 ? rows : 65535)), dim3(row_threads(F)), 0,
                                 static_cast<cudaStream_t>(stream), 1, p);
      });
    });
  });
}

extern "C" sp24_status sp24_gated_act_backward(sp24_dtype t, sp24_act act, int64_t rows, int64_t F, const void* dy, int64_t lddy,
                                               const void* g, int64_t ldg, const void* u, int64_t ldu, void* dg, int64_t lddg, void* du,
                                               int64_t lddu, void* stream) {
  SP24_RETURN_IF(!is_float_type(t), SP24_ERR_DTYPE);
  SP24_RETURN_IF(!is_act(act) || (!u && du), SP24_ERR_UNSUPPORTED);
  SP24_RETURN_IF(rows < 0 || F < 1 || F > kMostColumns, SP24_ERR_SHAPE);
  if (rows == 0) return SP24_OK;
  SP24_RETURN_IF(!dy || !g || !dg || (u && !du), SP24_ERR_NULL);
  SP24_RETURN_IF(!row_fits(rows, F, lddy) || !row_fits(rows, F, ldg) || (u && !row_fits(rows, F, ldu)) || !row_fits(rows, F, lddg) ||
                     (du && !row_fits(rows, F, lddu)),
                 SP24_ERR_STRIDE);
  const size_t es = elem_bytes(t);
  SP24_RETURN_IF(!aligned(dy, es) || !aligned(g, es) || !aligned(u, es) || !aligned(dg, es) || !aligned(du, es), SP24_ERR_ALIGN);
  const sp24_status st = check_arch();
  if (st != SP24_OK) return st;
  const GatedGradParams p = {rows, F, dy, g, u, dg, du, lddy, ldg, ldu, lddg, lddu};
  const int64_t across = (F + 255) / 256;
  return with_float_type(t, [&](auto type) {
    using T = typename decltype(type)::type;
    return with_act(act, [&](auto a) {
      return launch_overlapped(gated_act_grad_kernel<T, decltype(a)::value>, dim3((unsigned)(across < 65535 ? across : 65535), (unsigned)(rows < 32768 ? rows : 32768)), dim3(256), 0,
                               static_cast<cudaStream_t>(stream), 1, p);
    });
  });
}
