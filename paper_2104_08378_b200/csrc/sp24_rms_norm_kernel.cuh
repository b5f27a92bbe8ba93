// Kernels of the root-mean-square norm with the residual's addition and 8-bit results, and of its gradient.
#pragma once

#include "sp24_rms_norm.cuh"

namespace sp24 {
namespace {

// Rows of up to kMostTeamVectors vectors: a team of threads to a row, which holds it in registers, and the weight for all its rows.  One pass: the
// team's next row (without a residual the next two, in as many registers) is on its way while this one is reduced, multiplied and
// stored.  n = h rstd w with rstd from the row's sum of squares; 8-bit rows need no second reduction, since max |n| = rstd max |h w|.
// Bound by HBM: bf16 8192 x 12288 with residual -> e4m3 111 us = 6.35 TB/s, -> bf16 125 us = 6.45 TB/s (a copy: 6.5); a block to a row and two passes
// took 427.  Short calls are a launch: bf16 32 x 4096 2.1 us.  (One block of up to 1024 threads to an SM and the next row in registers instead of more blocks:
// what is on its way does not depend on where the teams stand.)
template <typename T, typename OUT, typename W, int V, bool RESIDUAL, bool WHOLE>
__global__ void __launch_bounds__(team_threads(V), 1) rms_norm_rows_kernel(const NormParams p) {
  constexpr int N = kVector<T>, kWords = sizeof(W) / sizeof(T);  // 16-byte words of a vector's weights
  __shared__ RowSums sums;
  int turn = 0;
  const int tx = threadIdx.x, team = blockDim.x;
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  wait_for_stream();
  uint4 a[V], b[V], w[V][kWords];  // a row and its residual, or two rows
  auto shift = [&](int64_t row) { return WHOLE ? 0 : shift_of<OUT, N>(static_cast<const OUT*>(p.y) + row * p.ldy); };
  auto fetch = [&](const void* from, int64_t ld, int64_t row, uint4 (&to)[V]) {
    if (row >= p.rows) return;
    const T* at = static_cast<const T*>(from) + row * ld;
#pragma unroll
    for (int v = 0; v < V; ++v) to[v] = load_vector<WHOLE>(at, tx + v * team, (int)p.K, shift(row));
  };
  // the weights of a row's vectors: those of all rows are the same if they are WHOLE
  auto fetch_weights = [&](int shift) {
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int i = 0; i < kWords; ++i) {
        Pairs<W> one;
#pragma unroll
        for (int n = 0; n < kVector<W> / 2; ++n) one[n] = both(1.f);
        w[v][i] = p.weight ? load_vector<WHOLE>(static_cast<const W*>(p.weight), (tx + v * team) * kWords + i, (int)p.K, shift) : pack<W>(one);
      }
  };
  int64_t base = (int64_t)blockIdx.x * blockDim.y;  // the first team's row: the warps of a block stay together
  fetch(p.x, p.ldx, base + threadIdx.y, a);
  if (RESIDUAL) fetch(p.residual, p.ldr, base + threadIdx.y, b);
  else fetch(p.x, p.ldx, base + step + threadIdx.y, b);
  if (WHOLE) fetch_weights(0);
  auto weighted = [&](int v, Pairs<T>& f) {  // f times the weights
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      Pairs<W> g;
      unpack<W>(w[v][i], g);
#pragma unroll
      for (int n = 0; n < kVector<W> / 2; ++n) f[i * (kVector<W> / 2) + n] = mul2(f[i * (kVector<W> / 2) + n], g[n]);
    }
  };
  // the row whose values are in x (and its residual in b), behind whose use the registers get the next ones
  auto one_row = [&](int64_t row, uint4 (&x)[V]) {
    const int K = row < p.rows ? (int)p.K : 0, s = row < p.rows ? shift(row) : 0;
    if (!WHOLE) fetch_weights(s);
    uint4 h[V];
    float sum[V], top = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float2 sum2 = both(0.f);
      h[v] = RESIDUAL ? add_packed<T>(x[v], b[v]) : x[v];
      Pairs<T> f;
      unpack<T>(h[v], f);
#pragma unroll
      for (int n = 0; n < N / 2; ++n) sum2 = fma2(f[n], f[n], sum2);
      sum[v] = sum2.x + sum2.y;
      if (is_code<OUT>) {
        weighted(v, f);
#pragma unroll
        for (int n = 0; n < N / 2; ++n) top = max_abs(top, f[n].x, f[n].y);
      }
    }
    fetch(p.x, p.ldx, row + (RESIDUAL ? step : 2 * step), x);
    if (RESIDUAL) {
      fetch(p.residual, p.ldr, row + step, b);
      if (p.h) {
        T* ph = static_cast<T*>(p.h) + row * p.ldh;
#pragma unroll
        for (int v = 0; v < V; ++v) store_vector<WHOLE>(ph, tx + v * team, K, s, h[v]);
      }
    }
    sums.reduce<true, is_code<OUT>>(sum, top, turn);
    const float rstd = rsqrtf(sum[0] / (float)p.K + p.eps);
    if (tx == 0 && K && p.rstd) p.rstd[row] = rstd;
    float factor = rstd;
    if (is_code<OUT>) {
      const float scale = row_scale<OUT>(top, rstd, &factor);
      if (tx == 0 && K) p.scale[row] = scale;
    }
    OUT* py = static_cast<OUT*>(p.y) + row * p.ldy;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      Pairs<T> f;
      unpack<T>(h[v], f);
      if (is_code<OUT>) weighted(v, f);
#pragma unroll
      for (int n = 0; n < N / 2; ++n) f[n] = mul2(f[n], both(factor));
      if (!is_code<OUT>) weighted(v, f);
      if constexpr (is_code<OUT>) store_codes<WHOLE, OUT>(py, tx + v * team, K, s, f);
      else store_vector<WHOLE>(py, tx + v * team, K, s, pack<T>(f));
    }
  };
  for (; base < p.rows; base += step) {
    one_row(base + threadIdx.y, a);
    if (!RESIDUAL) {
      base += step;
      if (base < p.rows) one_row(base + threadIdx.y, b);
    }
  }
}

// Longer rows: a block to a row, each thread with its first kKept vectors of h in registers (rows of up to 4096 vectors) and the others read twice, the second time
// from the caches.
constexpr int kKept = 4;
template <typename T, typename OUT>
__global__ void __launch_bounds__(1024, 1) rms_norm_kernel(const NormParams p) {
  constexpr int P = kVector<T> / 2;
  __shared__ RowSums sums;
  int turn = 0;
  const int K = (int)p.K;
  wait_for_stream();
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x) {
    const T* x = static_cast<const T*>(p.x) + row * p.ldx;
    const T* r = p.residual ? static_cast<const T*>(p.residual) + row * p.ldr : nullptr;
    T* h = p.h ? static_cast<T*>(p.h) + row * p.ldh : nullptr;
    OUT* y = static_cast<OUT*>(p.y) + row * p.ldy;
    const int shift = shift_of<OUT, kVector<T>>(y), vectors = (shift + K + kVector<T> - 1) / kVector<T>;
    auto value = [&](int i) {
      const uint4 a = load_vector<false>(x, i, K, shift);
      return r ? add_packed<T>(a, load_vector<false>(r, i, K, shift)) : a;
    };
    auto weighted = [&](int i, Pairs<T>& f) {
      if (!p.weight) return;
      Pairs<T> w;
      if (p.weight_f32 && sizeof(T) == 2) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          Pairs<float> half;
          unpack<float>(load_vector<false>(static_cast<const float*>(p.weight), 2 * i + q, K, shift), half);
          w[q * (P / 2)] = half[0];
          w[q * (P / 2) + P / 2 - 1] = half[1];
        }
      } else {
        unpack<T>(load_vector<false>(static_cast<const T*>(p.weight), i, K, shift), w);
      }
#pragma unroll
      for (int n = 0; n < P; ++n) f[n] = mul2(f[n], w[n]);
    };
    uint4 kept[kKept];
    float sum[2], top = 0.f;  // of the first vector, and of the others: of rows of 64 groups of vectors the same order as the teams'
    float2 sum2 = both(0.f);
    auto count = [&](int i, const uint4& v) {
      Pairs<T> f;
      unpack<T>(v, f);
#pragma unroll
      for (int n = 0; n < P; ++n) sum2 = fma2(f[n], f[n], sum2);
      if (is_code<OUT>) {
        weighted(i, f);
#pragma unroll
        for (int n = 0; n < P; ++n) top = max_abs(top, f[n].x, f[n].y);
      }
    };
#pragma unroll
    for (int v = 0; v < kKept; ++v) kept[v] = value(threadIdx.x + v * 1024);
    count(threadIdx.x, kept[0]);
    sum[0] = sum2.x + sum2.y;
    sum2 = both(0.f);
#pragma unroll
    for (int v = 1; v < kKept; ++v) count(threadIdx.x + v * 1024, kept[v]);
    for (int i = threadIdx.x + kKept * 1024; i < vectors; i += 1024) count(i, value(i));
    sum[1] = sum2.x + sum2.y;
    sums.reduce<true, is_code<OUT>>(sum, top, turn);
    const float rstd = rsqrtf(sum[0] / (float)p.K + p.eps);
    if (threadIdx.x == 0 && p.rstd) p.rstd[row] = rstd;
    float factor = rstd;
    if (is_code<OUT>) {
      const float scale = row_scale<OUT>(top, rstd, &factor);
      if (threadIdx.x == 0) p.scale[row] = scale;
    }
    auto store = [&](int i, const uint4& v) {
      Pairs<T> f;
      unpack<T>(v, f);
      if (is_code<OUT>) weighted(i, f);
#pragma unroll
      for (int n = 0; n < P; ++n) f[n] = mul2(f[n], both(factor));
      if (!is_code<OUT>) weighted(i, f);
      if (h) store_vector<false>(h, i, K, shift, v);
      if constexpr (is_code<OUT>) store_codes<false, OUT>(y, i, K, shift, f);
      else store_vector<false>(y, i, K, shift, pack<T>(f));
    };
#pragma unroll
    for (int v = 0; v < kKept; ++v) store(threadIdx.x + v * 1024, kept[v]);
    for (int i = threadIdx.x + kKept * 1024; i < vectors; i += 1024) store(i, value(i));
  }
}

// Rows of up to kMostTeamVectors vectors: a team of threads to a row, with the weight and the team's part of dweight in registers for all
// its rows.  AHEAD: the team's next row is on its way from before this one's work to the end of it, in registers of its own (two sets in
// turn).  At the end the block adds its teams' parts up, in an order that their number fixes.
// dx = rstd (v - h rstd^2 mean(v h)) + dh with v = dy w: one reduction to a row.  Bound by HBM: bf16 8192 x 8192 with dh 89 us = 6.0 TB/s (single set of
// registers 123, two passes 498); 512 threads of 123 registers are enough because 49 KB are on their way all the time.  512 x 4096 8.7 us, two launches.
constexpr int kAheadThreads = 512;
template <typename T, typename W, int V, bool AHEAD, bool WHOLE>
__global__ void __launch_bounds__(AHEAD ? kAheadThreads : team_threads(V), 1) rms_norm_grad_rows_kernel(const NormGradParams p) {
  constexpr int P = kVector<T> / 2, kWords = sizeof(W) / sizeof(T), PW = kVector<W> / 2;
  __shared__ RowSums sums;
  extern __shared__ float4 parts[];  // K rounded up to vectors, a row for each team of whole warps or for each warp
  int turn = 0;
  const int tx = threadIdx.x, team = blockDim.x, K = (int)p.K;
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  const float over_k = 1.f / (float)p.K;
  wait_for_stream();
  struct Row {
    uint4 dy[V], h[V], dh[V];
    float rstd;
  };
  auto fetch = [&](const void* from, int64_t ld, int64_t row, uint4 (&to)[V]) {
    const T* at = static_cast<const T*>(from) + row * ld;
#pragma unroll
    for (int v = 0; v < V; ++v) to[v] = load_vector<WHOLE>(at, tx + v * team, K, 0);  // (dweight's sums stay with their columns: no shift)
  };
  auto fetch_row = [&](int64_t row, Row& to) {
    if (row >= p.rows) return;
    to.rstd = p.rstd[row];
    fetch(p.dy, p.lddy, row, to.dy);
    fetch(p.h, p.ldh, row, to.h);
    if (p.dh) fetch(p.dh, p.lddh, row, to.dh);
  };
  Row a = {}, b = {};
  int64_t base = (int64_t)blockIdx.x * blockDim.y;  // the first team's row: the warps of a block stay together
  fetch_row(base + threadIdx.y, a);
  uint4 w[V][kWords];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      Pairs<W> one;
#pragma unroll
      for (int n = 0; n < PW; ++n) one[n] = both(1.f);
      w[v][i] = p.weight ? load_vector<WHOLE>(static_cast<const W*>(p.weight), (tx + v * team) * kWords + i, K, 0) : pack<W>(one);
    }
  auto weighted = [&](int v, Pairs<T>& f) {  // f times the weights
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
      Pairs<W> g;
      unpack<W>(w[v][i], g);
#pragma unroll
      for (int n = 0; n < PW; ++n) f[i * PW + n] = mul2(f[i * PW + n], g[n]);
    }
  };
  Pairs<T> acc[V];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int n = 0; n < P; ++n) acc[v][n] = both(0.f);
  auto one_row = [&](int64_t row, Row& x, Row& next) {
    const bool live = row < p.rows;
    if (AHEAD) fetch_row(row + step, next);
    const float r = x.rstd;
    float sum[V], unused = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      float2 sum2 = both(0.f);
      Pairs<T> g, f;
      unpack<T>(x.dy[v], g);
      unpack<T>(x.h[v], f);
#pragma unroll
      for (int n = 0; n < P; ++n) {
        const float2 s = mul2(g[n], f[n]);
        if (live) acc[v][n] = fma2(s, both(r), acc[v][n]);
      }
      weighted(v, g);
#pragma unroll
      for (int n = 0; n < P; ++n) sum2 = fma2(g[n], f[n], sum2);
      sum[v] = sum2.x + sum2.y;
    }
    sums.reduce<true, false>(sum, unused, turn);
    const float along = -sum[0] * over_k * r * r;
    T* dx = static_cast<T*>(p.dx) + row * p.lddx;
    uint4 out[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      Pairs<T> g, f, d;
      unpack<T>(x.dy[v], g);
      unpack<T>(x.h[v], f);
      unpack<T>(x.dh[v], d);
      weighted(v, g);
#pragma unroll
      for (int n = 0; n < P; ++n) g[n] = fma2(fma2(f[n], both(along), g[n]), both(r), d[n]);
      out[v] = pack<T>(g);
    }
    if (!AHEAD) fetch_row(row + step, x);
#pragma unroll
    for (int v = 0; v < V; ++v) store_vector<WHOLE>(dx, tx + v * team, live ? K : 0, 0, out[v]);
  };
  for (; base < p.rows; base += step) {
    one_row(base + threadIdx.y, a, b);
    if (AHEAD) {
      base += step;
      if (base < p.rows) one_row(base + threadIdx.y, b, a);
    }
  }
  if (!p.partial) return;
  const int vectors = (K + 2 * P - 1) / (2 * P), thread = threadIdx.y * team + tx;
  if (team < 32) {  // the teams of a warp: lanes `team` apart have the same columns
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int n = 0; n < P; ++n)
        for (int i = 16; i >= team; i >>= 1) {
          acc[v][n].x += __shfl_xor_sync(~0u, acc[v][n].x, i);
          acc[v][n].y += __shfl_xor_sync(~0u, acc[v][n].y, i);
        }
  }
  const int slots = team < 32 ? (int)blockDim.y * team / 32 : (int)blockDim.y, slot = team < 32 ? thread / 32 : (int)threadIdx.y;
  constexpr int kQuads = P / 2;  // 16-byte groups of a vector's sums
  if (team >= 32 || (thread & 31) < team) {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int i = tx + v * team;
#pragma unroll
      for (int q = 0; q < kQuads; ++q)
        if (i < vectors) parts[(slot * kQuads + q) * vectors + i] = make_float4(acc[v][2 * q].x, acc[v][2 * q].y, acc[v][2 * q + 1].x, acc[v][2 * q + 1].y);
    }
  }
  __syncthreads();
  float* to = p.partial + (int64_t)blockIdx.x * p.K;
  for (int c = thread; c < vectors * kQuads; c += team * blockDim.y) {
    const int i = c / kQuads, q = c % kQuads;
    float4 s = parts[q * vectors + i];
    for (int t = 1; t < slots; ++t) {
      const float4 o = parts[(t * kQuads + q) * vectors + i];
      s.x += o.x; s.y += o.y; s.z += o.z; s.w += o.w;
    }
    const int k = i * 2 * P + q * 4;
    if (k < K) to[k] = s.x;
    if (k + 1 < K) to[k + 1] = s.y;
    if (k + 2 < K) to[k + 2] = s.z;
    if (k + 3 < K) to[k + 3] = s.w;
  }
}

// Longer rows: a block to a row, two passes over it (the second from the caches).  The block's part of dweight: of each thread's first kKept vectors in
// registers (rows of up to 4096 vectors), of the others in the workspace.
template <typename T>
__global__ void __launch_bounds__(1024, 1) rms_norm_grad_kernel(const NormGradParams p) {
  constexpr int N = kVector<T>, P = N / 2;
  __shared__ RowSums sums;
  int turn = 0;
  const int K = (int)p.K, vectors = (K + N - 1) / N;
  wait_for_stream();
  float* part = p.partial ? p.partial + blockIdx.x * p.K : nullptr;
  Pairs<T> acc[kKept];
#pragma unroll
  for (int v = 0; v < kKept; ++v)
#pragma unroll
    for (int n = 0; n < P; ++n) acc[v][n] = both(0.f);
  bool first = true;
  for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, first = false) {
    const T* dy = static_cast<const T*>(p.dy) + row * p.lddy;
    const T* h = static_cast<const T*>(p.h) + row * p.ldh;
    const T* dh = p.dh ? static_cast<const T*>(p.dh) + row * p.lddh : nullptr;
    T* dx = static_cast<T*>(p.dx) + row * p.lddx;
    const float rstd = p.rstd[row];
    auto load = [&](int i, Pairs<T>& g, Pairs<T>& f) {
      unpack<T>(load_vector<false>(dy, i, K, 0), g);
      unpack<T>(load_vector<false>(h, i, K, 0), f);
    };
    auto weighted = [&](int i, Pairs<T>& f) {
      if (!p.weight) return;
#pragma unroll
      for (int n = 0; n < P; ++n) {
        const int k = i * N + 2 * n;
        f[n] = mul2(f[n], make_float2(k < K ? load_weight<T>(p.weight, p.weight_f32, k) : 0.f, k + 1 < K ? load_weight<T>(p.weight, p.weight_f32, k + 1) : 0.f));
      }
    };
    float2 sum2 = both(0.f);
#pragma unroll 4
    for (int i = threadIdx.x; i < vectors; i += 1024) {
      Pairs<T> g, f;
      load(i, g, f);
      weighted(i, g);
#pragma unroll
      for (int n = 0; n < P; ++n) sum2 = fma2(g[n], f[n], sum2);
    }
    float sum[1] = {sum2.x + sum2.y}, unused = 0.f;
    sums.reduce<true, false>(sum, unused, turn);
    const float along = -sum[0] / (float)p.K * rstd * rstd;
    auto finish = [&](int i, Pairs<T>& g, const Pairs<T>& f) {
      Pairs<T> d = {};
      if (dh) unpack<T>(load_vector<false>(dh, i, K, 0), d);
      weighted(i, g);
#pragma unroll
      for (int n = 0; n < P; ++n) g[n] = fma2(fma2(f[n], both(along), g[n]), both(rstd), d[n]);
      store_vector<false>(dx, i, K, 0, pack<T>(g));
    };
#pragma unroll
    for (int v = 0; v < kKept; ++v) {
      const int i = threadIdx.x + v * 1024;
      Pairs<T> g, f;
      load(i, g, f);
#pragma unroll
      for (int n = 0; n < P; ++n) acc[v][n] = fma2(mul2(g[n], f[n]), both(rstd), acc[v][n]);
      finish(i, g, f);
    }
    for (int i = threadIdx.x + kKept * 1024; i < vectors; i += 1024) {
      Pairs<T> g, f;
      load(i, g, f);
      if (part) {
#pragma unroll
        for (int n = 0; n < P; ++n) {
          const int k = i * N + 2 * n;
          if (k < K) part[k] = fmaf(g[n].x * f[n].x, rstd, first ? 0.f : part[k]);
          if (k + 1 < K) part[k + 1] = fmaf(g[n].y * f[n].y, rstd, first ? 0.f : part[k + 1]);
        }
      }
      finish(i, g, f);
    }
  }
  if (!part) return;
#pragma unroll
  for (int v = 0; v < kKept; ++v)
#pragma unroll
    for (int n = 0; n < P; ++n) {
      const int k = (threadIdx.x + v * 1024) * N + 2 * n;
      if (k < K) part[k] = acc[v][n].x;
      if (k + 1 < K) part[k + 1] = acc[v][n].y;
    }
}

}  // namespace

template <typename T>
sp24_status launch_rms_norm(sp24_dtype out_type, const NormParams& p, bool whole, cudaStream_t s) {
  const int64_t vectors = row_vectors(p.K, sizeof(T), whole);
  return with_out_type<T>(out_type, [&](auto out) {
    using OUT = typename decltype(out)::type;
    if (vectors <= kMostTeamVectors) {
      const TeamLaunch at(p.rows, vectors, 8);  // (bf16 512 x 4096 with one vector and two: 4.4, 5.7 us; 1024 rows 7.6, 8.0; 8192 rows 44.6, 43.4)
      auto launch = [&](auto weight_t) {
        using W = typename decltype(weight_t)::type;
        const auto kernel = with_flags(
            [](auto four, auto two, auto with_residual, auto whole) {
              return rms_norm_rows_kernel<T, OUT, W, four.value ? 4 : two.value ? 2 : 1, with_residual.value, whole.value>;
            },
            at.v == 4, at.v >= 2, p.residual != nullptr, whole);
        return launch_overlapped(kernel, at.grid, at.block, 0, s, 1, p);
      };
      return p.weight && p.weight_f32 ? launch(TypeOf<float>{}) : launch(TypeOf<T>{});
    }
    return launch_overlapped(rms_norm_kernel<T, OUT>, dim3((unsigned)(p.rows < 65535 ? p.rows : 65535)), dim3(1024), 0,
                             s, 1, p);
  });
}

template <typename T>
sp24_status launch_rms_norm_grad(const NormGradParams& p, bool whole, int64_t& blocks, cudaStream_t s) {
  const int64_t vectors = row_vectors(p.K, sizeof(T), true);
  if (vectors <= kMostTeamVectors) {
    const TeamLaunch at(p.rows, vectors, 2, kAheadThreads);  // (bf16 512 x 4096 with one vector and two: 9.4, 8.7 us)
    blocks = at.grid.x;
    const int slots = at.block.x < 32 ? (int)(at.block.x * at.block.y / 32) : (int)at.block.y;
    const size_t smem = p.partial ? (size_t)slots * vectors * kVector<T> * sizeof(float) : 0;  // (at most 64 KB: V vectors for each thread)
    auto launch = [&](auto weight_t) {
      using W = typename decltype(weight_t)::type;
      const auto kernel = at.v == 2 && vectors <= 2 * kAheadThreads
                              ? (whole ? rms_norm_grad_rows_kernel<T, W, 2, true, true> : rms_norm_grad_rows_kernel<T, W, 2, true, false>)
                              : with_flags([](auto four, auto two, auto whole) { return rms_norm_grad_rows_kernel<T, W, four.value ? 4 : two.value ? 2 : 1, false, whole.value>; },
                                           at.v == 4, at.v >= 2, whole);
      if (smem > 48 * 1024 - sizeof(RowSums)) SP24_CUDA_CHECK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 64 * 1024));
      return launch_overlapped(kernel, at.grid, at.block, smem, s, 1, p);
    };
    return p.weight && p.weight_f32 ? launch(TypeOf<float>{}) : launch(TypeOf<T>{});
  }
  blocks = p.rows < sm_count() ? p.rows : sm_count();
  return launch_overlapped(rms_norm_grad_kernel<T>, dim3((unsigned)blocks), dim3(1024), 0, s, 1, p);
}

}  // namespace sp24
