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
};

// act(g) * u of a vector
template <typename T>
__device__ __forceinline__ void gated_vector(int act, const uint4& g, const uint4& u, bool gated, Pairs<T>& y) {
  constexpr int P = kVector<T> / 2;
  unpack<T>(g, y);
  device_with_act(act, [&](auto a) {
#pragma unroll
    for (int n = 0; n < P; ++n) y[n] = act_value<decltype(a)::value>(y[n]);
  });
  if (gated) {
    Pairs<T> f;
    unpack<T>(u, f);
#pragma unroll
    for (int n = 0; n < P; ++n) y[n] = mul2(y[n], f[n]);
  }
}

// Rows of up to kMostTeamVectors vectors: a team of threads to a row, whose results it holds in registers until their maximum is known.
// AHEAD: the team's next row is on its way from before this one's activations to the end of it, in registers of its own (two sets in
// turn): the exponentials and reciprocals take half as long as the memory does.  Else it sets out behind them, and more teams, each at another
// place of its row, hide that.
// Bound by the special-function units (52 % busy: an exponential and a reciprocal for each value), the ALU (46 %) and HBM, which the barrier of 8-bit rows keeps from
// overlapping wholly: silu bf16 8192 x 12288 -> e4m3 85 us = 5.9 TB/s, -> bf16 92 us = 6.5 TB/s, gelu -> int8 104 us; two passes took 455.
constexpr int many_threads(int v) { return v == 2 ? 1024 : 768; }
template <typename T, typename OUT, int V, bool AHEAD, bool WHOLE>
__global__ void __launch_bounds__(AHEAD ? team_threads(V) : many_threads(V), 1) gated_act_rows_kernel(const GatedParams p) {
  constexpr int N = kVector<T>, P = N / 2;
  __shared__ RowSums sums;
  int turn = 0;
  const int tx = threadIdx.x, team = blockDim.x, F = (int)p.F;
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  const bool gated = p.u != nullptr;
  wait_for_stream();
  struct Row {
    uint4 g[V], u[V];
  };
  auto shift = [&](int64_t row) { return WHOLE ? 0 : shift_of<OUT, N>(static_cast<const OUT*>(p.y) + row * p.ldy); };
  auto fetch = [&](int64_t row, Row& to) {
    if (row >= p.rows) return;
    const int s = shift(row);
    const T* pg = static_cast<const T*>(p.g) + row * p.ldg;
    const T* pu = static_cast<const T*>(p.u) + row * p.ldu;
#pragma unroll
    for (int v = 0; v < V; ++v) to.g[v] = load_vector<WHOLE>(pg, tx + v * team, F, s);
    if (gated) {
#pragma unroll
      for (int v = 0; v < V; ++v) to.u[v] = load_vector<WHOLE>(pu, tx + v * team, F, s);
    }
  };
  auto one_row = [&](int64_t row, Row& x, Row& next) {
    const int K = row < p.rows ? F : 0, s = row < p.rows ? shift(row) : 0;
    if (AHEAD) fetch(row + step, next);
    Pairs<T> y[V];
    float top = 0.f, unused[1] = {}, inv = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      gated_vector<T>(p.act, x.g[v], x.u[v], gated, y[v]);
      if (is_code<OUT>) {
#pragma unroll
        for (int n = 0; n < P; ++n) top = max_abs(top, y[v][n].x, y[v][n].y);
      }
    }
    if (!AHEAD) fetch(row + step, x);
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
        store_codes<WHOLE, OUT>(py, tx + v * team, K, s, y[v]);
      } else {
        store_vector<WHOLE>(py, tx + v * team, K, s, pack<T>(y[v]));
      }
    }
  };
  Row a = {}, b = {};
  int64_t base = (int64_t)blockIdx.x * blockDim.y;  // the first team's row: the warps of a block stay together
  fetch(base + threadIdx.y, a);
  for (; base < p.rows; base += step) {
    one_row(base + threadIdx.y, a, b);
    if (AHEAD) {
      base += step;
      if (base < p.rows) one_row(base + threadIdx.y, b, a);
    }
  }
}

// Longer rows: a block to a row, each thread with its first kKept vectors' results in registers (rows of up to 4096 vectors) and the others computed twice for
// 8-bit results, the second time from the caches.
constexpr int kKept = 4;
template <typename T, typename OUT>
__global__ void __launch_bounds__(1024, 1) gated_act_kernel(const GatedParams p) {
  constexpr int P = kVector<T> / 2;
  __shared__ RowSums sums;
  int turn = 0;
  const int K = (int)p.F;
  wait_for_stream();
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const T* g = static_cast<const T*>(p.g) + row * p.ldg;
    const T* u = p.u ? static_cast<const T*>(p.u) + row * p.ldu : nullptr;
    OUT* y = static_cast<OUT*>(p.y) + row * p.ldy;
    const int shift = shift_of<OUT, kVector<T>>(y), vectors = (shift + K + kVector<T> - 1) / kVector<T>;
    auto value = [&](int i, Pairs<T>& f) {
      const uint4 a = load_vector<false>(g, i, K, shift);
      gated_vector<T>(p.act, a, u ? load_vector<false>(u, i, K, shift) : a, u != nullptr, f);
    };
    Pairs<T> kept[kKept];
    float top = 0.f, unused[1] = {}, inv = 0.f;
    auto count = [&](const Pairs<T>& f) {
#pragma unroll
      for (int n = 0; n < P; ++n) top = max_abs(top, f[n].x, f[n].y);
    };
#pragma unroll
    for (int v = 0; v < kKept; ++v) {
      value(threadIdx.x + v * 1024, kept[v]);
      if (is_code<OUT>) count(kept[v]);
    }
    if (is_code<OUT>) {
      for (int i = threadIdx.x + kKept * 1024; i < vectors; i += 1024) {
        Pairs<T> f;
        value(i, f);
        count(f);
      }
      sums.reduce<false, true>(unused, top, turn);
      const float scale = row_scale<OUT>(finite_or_nan(top), 1.f, &inv);
      if (threadIdx.x == 0) p.scale[row] = scale;
    }
    auto store = [&](int i, Pairs<T>& f) {
      if constexpr (is_code<OUT>) {
#pragma unroll
        for (int n = 0; n < P; ++n) f[n] = mul2(f[n], both(inv));
        store_codes<false, OUT>(y, i, K, shift, f);
      } else {
        store_vector<false>(y, i, K, shift, pack<T>(f));
      }
    };
#pragma unroll
    for (int v = 0; v < kKept; ++v) store(threadIdx.x + v * 1024, kept[v]);
    for (int i = threadIdx.x + kKept * 1024; i < vectors; i += 1024) {
      Pairs<T> f;
      value(i, f);
      store(i, f);
    }
  }
}

struct GatedGradParams {
  int64_t rows, F;
  const void *dy, *g, *u;
  void *dg, *du;
  int64_t lddy, ldg, ldu, lddg, lddu;
  int32_t act;
};

// Element by element: two vectors to a thread, all their loads before the first use.  Bound by HBM: bf16 4096 x 8192 51 us = 6.6 TB/s with any activation
// (an element to a thread 214); rows that lie otherwise than the results' take two words and a shift for each vector: f16 4099 x 5461 with GELU 57 us, 3.9 TB/s.
template <typename T, bool WHOLE>
__global__ void __launch_bounds__(kThreads) gated_act_grad_kernel(const GatedGradParams p) {
  constexpr int P = kVector<T> / 2, V = 2;
  const int tx = threadIdx.x, F = (int)p.F, i0 = blockIdx.x * (V * blockDim.x) + tx;
  const bool gated = p.u != nullptr;
  wait_for_stream();
  for (int64_t base = (int64_t)blockIdx.y * blockDim.y; base < p.rows; base += (int64_t)gridDim.y * blockDim.y) {
    const int64_t row = base + threadIdx.y;
    if (row >= p.rows) break;
    const int s = WHOLE ? 0 : shift_of<T, kVector<T>>(static_cast<const T*>(p.dg) + row * p.lddg);
    const T *pdy = static_cast<const T*>(p.dy) + row * p.lddy, *pg = static_cast<const T*>(p.g) + row * p.ldg, *pu = static_cast<const T*>(p.u) + row * p.ldu;
    Words<WHOLE> dy[V], g[V], u[V] = {};
#pragma unroll
    for (int v = 0; v < V; ++v) load_words<WHOLE>(dy[v], pdy, i0 + v * (int)blockDim.x, F, s);
#pragma unroll
    for (int v = 0; v < V; ++v) load_words<WHOLE>(g[v], pg, i0 + v * (int)blockDim.x, F, s);
    if (gated) {
#pragma unroll
      for (int v = 0; v < V; ++v) load_words<WHOLE>(u[v], pu, i0 + v * (int)blockDim.x, F, s);
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int i = i0 + v * (int)blockDim.x;
      Pairs<T> d, f, w, dg, du;
      unpack<T>(vector_of<WHOLE>(dy[v], pdy, i, F, s), d);
      unpack<T>(vector_of<WHOLE>(g[v], pg, i, F, s), f);
      unpack<T>(vector_of<WHOLE>(u[v], pu, i, F, s), w);
      device_with_act(p.act, [&](auto a) {
#pragma unroll
        for (int n = 0; n < P; ++n) {
          float2 slope;
          du[n] = mul2(act_and_slope<decltype(a)::value>(f[n], &slope), d[n]);
          dg[n] = mul2(gated ? mul2(d[n], w[n]) : d[n], slope);
        }
      });
      store_vector<WHOLE>(static_cast<T*>(p.dg) + row * p.lddg, i, F, s, pack<T>(dg));
      if (gated) store_vector<WHOLE>(static_cast<T*>(p.du) + row * p.lddu, i, F, s, pack<T>(du));
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
  const GatedParams p = {rows, F, g, u, y, scale, ldg, ldu, ldy, (int)act};
  const bool whole = F * es % 16 == 0 && whole_rows(g, rows, ldg, es, 16) && whole_rows(u, rows, ldu, es, 16) && whole_rows(y, rows, ldy, os, 16 / es * os);
  const int64_t vectors = row_vectors(F, es, whole);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return with_float_type(t, [&](auto type) {
    using T = typename decltype(type)::type;
    return with_out_type<T>(out_type, [&](auto out) {
      using OUT = typename decltype(out)::type;
      if (vectors > kMostTeamVectors) return launch_overlapped(gated_act_kernel<T, OUT>, dim3((unsigned)(rows < 65535 ? rows : 65535)), dim3(1024), 0, s, 1, p);
      // Where a row's team leaves threads out (768 of them with two vectors and the next row ahead), more teams without it: two vectors and 1024 threads,
      // if that puts half as many threads again to work (silu bf16 8192 x 8192 -> e4m3 69.1, 57.5 us, x 5120 39.1, 37.9; not x 6144 43.6, 47.5,
      // x 4096 29.7, 29.3); for 8-bit results of rows of one team, which all wait for the maximum, two teams with four vectors if there are many
      // rows (8192 x 12288 89.7, 85.5, x 9216 77.5, 74.3; not 1024 x 12288 13.5, 15.0, nor -> bf16 92.5, 95.4).
      const int64_t team = ((vectors + 1) / 2 + 31) / 32 * 32;
      const bool many = vectors <= 1024 && 2 * (1024 / team) >= 3 * (team_threads(2) / team);
      if constexpr (is_code<OUT>)
        if (vectors > 1024 && vectors <= 2 * many_threads(4) && rows >= 32 * (int64_t)sm_count()) {
          const unsigned of_four = (unsigned)((vectors + 3) / 4 + 31) / 32 * 32;
          return launch_overlapped(whole ? gated_act_rows_kernel<T, OUT, 4, false, true> : gated_act_rows_kernel<T, OUT, 4, false, false>,
                                   dim3((unsigned)sm_count()), dim3(of_four, many_threads(4) / of_four), 0, s, 1, p);
        }
      const TeamLaunch at(rows, vectors, 2, many ? many_threads(2) : team_threads(2));
      const auto kernel = at.v == 2 && many
                              ? (whole ? gated_act_rows_kernel<T, OUT, 2, false, true> : gated_act_rows_kernel<T, OUT, 2, false, false>)
                              : with_flags([](auto four, auto two, auto whole) { return gated_act_rows_kernel<T, OUT, four.value ? 4 : two.value ? 2 : 1, true, whole.value>; },
                                           at.v == 4, at.v >= 2, whole);
      return launch_overlapped(kernel, at.grid, at.block, 0, s, 1, p);
    });
  });
}

extern "C" sp24_status sp24_gated_act_backward(sp24_dtype t, sp24_act act, int64_t rows, int64_t F, const void* dy, int64_t lddy,
                                               const void* g, int64_t ldg, const void* u, int64_t ldu, void* dg, int64_t lddg, void* du,
                                               int64_t lddu, void* stream) {
  SP24_RETURN_IF(!is_float_type(t), SP24_ERR_DTYPE);
  SP24_RETURN_IF(!is_act(act) || (!u && du) || (du && du == dg), SP24_ERR_UNSUPPORTED);
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
  const GatedGradParams p = {rows, F, dy, g, u, dg, du, lddy, ldg, ldu, lddg, lddu, (int)act};
  const bool whole = F * es % 16 == 0 && whole_rows(dy, rows, lddy, es, 16) && whole_rows(g, rows, ldg, es, 16) && whole_rows(u, rows, ldu, es, 16) &&
                     whole_rows(dg, rows, lddg, es, 16) && whole_rows(du, rows, lddu, es, 16);
  const RowLaunch at(row_vectors(F, es, whole), rows, 2);
  return with_float_type(t, [&](auto type) {
    using T = typename decltype(type)::type;
    return launch_overlapped(whole ? gated_act_grad_kernel<T, true> : gated_act_grad_kernel<T, false>, at.grid, at.block, 0, static_cast<cudaStream_t>(stream), 1, p);
  });
}
