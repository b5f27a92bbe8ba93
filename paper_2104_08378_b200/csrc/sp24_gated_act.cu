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
  int32_t act;
  bool whole_g, whole_u, whole_y;  // rows at boundaries of vectors
};

// act(g) * u of a vector
template <typename T>
__device__ __forceinline__ void gated_vector(int act, const uint4& g, const uint4& u, bool gated, Pairs<T>& y) {
  constexpr int P = kVector<T> / 2;
  unpack<T>(g, y);
  device_with_act(act, [&](auto a) {
#pragma unroll
    for (int n = 0; n < P; ++n) y[n] = make_float2(act_value<decltype(a)::value>(y[n].x), act_value<decltype(a)::value>(y[n].y));
  });
  if (gated) {
    Pairs<T> f;
    unpack<T>(u, f);
#pragma unroll
    for (int n = 0; n < P; ++n) y[n] = mul2(y[n], f[n]);
  }
}

// Rows of up to kMostTeamVectors vectors: a team of threads to a row, whose results it holds in registers until their maximum is known.  The
// team's next row is on its way from before this one's activations to the end of it, in registers of its own (two sets in turn): the
// exponentials and reciprocals take half as long as the memory does.
template <typename T, typename OUT, int V, bool WHOLE>
__global__ void __launch_bounds__(team_threads(V), 1) gated_act_rows_kernel(const GatedParams p) {
  constexpr int P = kVector<T> / 2;
  __shared__ RowSums sums;
  int turn = 0;
  const int tx = threadIdx.x, team = blockDim.x, F = (int)p.F;
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  const bool gated = p.u != nullptr;
  wait_for_stream();
  struct Row {
    uint4 g[V], u[V];
  };
  auto fetch = [&](int64_t row, Row& to) {
    if (row >= p.rows) return;
    const T* pg = static_cast<const T*>(p.g) + row * p.ldg;
    const T* pu = static_cast<const T*>(p.u) + row * p.ldu;
#pragma unroll
    for (int v = 0; v < V; ++v) to.g[v] = load_vector<WHOLE>(pg, tx + v * team, F, p.whole_g);
    if (gated) {
#pragma unroll
      for (int v = 0; v < V; ++v) to.u[v] = load_vector<WHOLE>(pu, tx + v * team, F, p.whole_u);
    }
  };
  auto one_row = [&](int64_t row, const Row& x, Row& next) {
    const int K = row < p.rows ? F : 0;
    fetch(row + step, next);
    Pairs<T> y[V];
    float top = 0.f, unused = 0.f, inv = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      gated_vector<T>(p.act, x.g[v], x.u[v], gated, y[v]);
      if (is_code<OUT>) {
#pragma unroll
        for (int n = 0; n < P; ++n) top = max_abs(top, y[v][n].x, y[v][n].y);
      }
    }
    if (is_code<OUT>) {
      sums.reduce<false, true>(unused, top, turn);
      const float scale = row_scale<OUT>(finite_or_nan(top), 1.f, &inv);
      if (tx == 0 && K) p.scale[row] = scale;
    }
    OUT* py = static_cast<OUT*>(p.y) + row * p.ldy;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      if constexpr (is_code<OUT>) {
#pragma unroll
        for (int n = 0; n < P; ++n) y[v][n] = mul2(y[v][n], both(inv));
        store_codes<WHOLE, OUT>(py, tx + v * team, K, p.whole_y, y[v]);
      } else {
        store_vector<WHOLE>(py, tx + v * team, K, p.whole_y, pack<T>(y[v]));
      }
    }
  };
  Row a = {}, b = {};
  int64_t base = (int64_t)blockIdx.x * blockDim.y;  // the first team's row: the warps of a block stay together
  fetch(base + threadIdx.y, a);
  for (; base < p.rows; base += 2 * step) {
    one_row(base + threadIdx.y, a, b);
    if (base + step < p.rows) one_row(base + step + threadIdx.y, b, a);
  }
}

// Longer rows: a block to a row; for 8-bit results a pass before it for the row's maximum, behind which the caches have the row.
template <typename T, typename OUT>
__global__ void __launch_bounds__(1024, 1) gated_act_kernel(const GatedParams p) {
  constexpr int P = kVector<T> / 2;
  __shared__ RowSums sums;
  int turn = 0;
  const int K = (int)p.F, vectors = (K + kVector<T> - 1) / kVector<T>;
  wait_for_stream();
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const T* g = static_cast<const T*>(p.g) + row * p.ldg;
    const T* u = p.u ? static_cast<const T*>(p.u) + row * p.ldu : nullptr;
    OUT* y = static_cast<OUT*>(p.y) + row * p.ldy;
    auto value = [&](int i, Pairs<T>& f) {
      const uint4 a = load_vector<false>(g, i, K, p.whole_g);
      gated_vector<T>(p.act, a, u ? load_vector<false>(u, i, K, p.whole_u) : a, u != nullptr, f);
    };
    float inv = 0.f;
    if (is_code<OUT>) {
      float top = 0.f, unused = 0.f;
#pragma unroll 2
      for (int i = threadIdx.x; i < vectors; i += blockDim.x) {
        Pairs<T> f;
        value(i, f);
#pragma unroll
        for (int n = 0; n < P; ++n) top = max_abs(top, f[n].x, f[n].y);
      }
      sums.reduce<false, true>(unused, top, turn);
      const float scale = row_scale<OUT>(finite_or_nan(top), 1.f, &inv);
      if (threadIdx.x == 0) p.scale[row] = scale;
    }
#pragma unroll 2
    for (int i = threadIdx.x; i < vectors; i += blockDim.x) {
      Pairs<T> f;
      value(i, f);
      if constexpr (is_code<OUT>) {
#pragma unroll
        for (int n = 0; n < P; ++n) f[n] = mul2(f[n], both(inv));
        store_codes<false, OUT>(y, i, K, p.whole_y, f);
      } else {
        store_vector<false>(y, i, K, p.whole_y, pack<T>(f));
      }
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
  const size_t os = elem_bytes(out_type);
  const GatedParams p = {rows, F, g, u, y, scale, ldg, ldu, ldy, (int)act, whole_rows(g, rows, ldg, es, 16), !u || whole_rows(u, rows, ldu, es, 16),
                         whole_rows(y, rows, ldy, os, 16 / es * os)};
  const int64_t vectors = (F * (int64_t)es + 15) / 16;
  const bool whole = p.whole_g && p.whole_u && p.whole_y && F * es % 16 == 0;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return with_float_type(t, [&](auto type) {
    using T = typename decltype(type)::type;
    return with_out_type<T>(out_type, [&](auto out) {
      using OUT = typename decltype(out)::type;
      if (vectors > kMostTeamVectors) return launch_overlapped(gated_act_kernel<T, OUT>, dim3((unsigned)(rows < 65535 ? rows : 65535)), dim3(1024), 0, s, 1, p);
      const TeamLaunch at(rows, vectors);
      const auto kernel = with_flags([](auto four, auto two, auto whole) { return gated_act_rows_kernel<T, OUT, four.value ? 4 : two.value ? 2 : 1, whole.value>; },
                                     at.v == 4, at.v >= 2, whole);
      return launch_overlapped(kernel, at.grid, at.block, 0, s, 1, p);
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
