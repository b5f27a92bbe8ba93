// Gradient of the activation between a product and what follows it: dz = dy * act'(z), in both orders (the two products of a linear
// layer's gradient contract over different axes), and the bias's gradient, the sums of dz over tokens.
#include "sp24_act.cuh"
#include "sp24_ptx.cuh"
#include "sp24_rows.cuh"

namespace sp24 {
namespace {

constexpr int kTile = 64;

struct ActGradParams {
  int64_t rows, cols;
  const void *dy, *z;
  void *dz, *dzt;
  float* partial;  // sums over the rows of a tile (over_rows: [row tiles][cols]) or over its columns ([column tiles][rows]); or null
  int64_t lddy, ldz, lddz, lddzt;
  int32_t over_rows;
  const int32_t* offsets;  // see sp24_expert_act_backward
  int32_t experts;
};

// 16-bit types, all rows (of dzt too) whole vectors at 16-byte boundaries.  A block to a tile of 128 x 128 (rows of 256 bytes both ways; of 64 x 64 where those
// would leave SMs idle: 128 x 4096 5.4 -> 3.6 us), transposed on its way out of
// shared memory by ldmatrix.trans: the eight rows of matrix i are 8 j + 2 i + b (j = 0..3, b = 0, 1), which leaves lane 4 c + j with eight
// consecutive rows of column c, so that a warp stores eight segments of 64 bytes.  Unit u (16 bytes) of row m lies at
// u ^ (2 (m >> 3 & 3) + (m & 1)): the eight rows of a matrix are in different banks.
// dz = dy act'(z) is needed in both orders, and reading dy and z once for both is what the tile is for.  Bound by HBM and, with GELU, the arithmetic of the slope:
// bf16 4096 x 8192 with the bias 52 us = 5.1 TB/s (ReLU 46; by elements 125, tiles of 64 x 64 62); three blocks to an SM instead of two spill (75).
template <typename T, int ACT, int kWide>
__global__ void __launch_bounds__(4 * kWide) act_grad_tile_kernel(const ActGradParams p) {
  constexpr int kUnits = kWide / 8, kWideThreads = 4 * kWide;
  constexpr int kPasses = kWide * kUnits / kWideThreads, kRows = kWide / kPasses;
  __shared__ uint4 tile[kWide * kUnits];
  __shared__ float over[kWideThreads / 32][kWide];  // sums over the rows of each warp
  const int64_t col_tiles = (p.cols + kWide - 1) / kWide;
  const int64_t row0 = (int64_t)(blockIdx.x / col_tiles) * kWide, col0 = (int64_t)(blockIdx.x % col_tiles) * kWide;
  const int u = threadIdx.x % kUnits, m0 = threadIdx.x / kUnits, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int64_t c = col0 + 8 * u;
  wait_for_stream();
  uint4 dy[kPasses] = {}, z[kPasses] = {};
#pragma unroll
  for (int v = 0; v < kPasses; ++v)
    if (const int64_t r = row0 + m0 + kRows * v; r < p.rows && c < p.cols) dy[v] = ld_stream(static_cast<const T*>(p.dy) + r * p.lddy + c);
  if (ACT != SP24_ACT_NONE) {
#pragma unroll
    for (int v = 0; v < kPasses; ++v)
      if (const int64_t r = row0 + m0 + kRows * v; r < p.rows && c < p.cols) z[v] = ld_stream(static_cast<const T*>(p.z) + r * p.ldz + c);
  }
  Pairs<T> sums = {};
#pragma unroll
  for (int v = 0; v < kPasses; ++v) {
    const int m = m0 + kRows * v;
    const int64_t r = row0 + m;
    Pairs<T> d, f;
    unpack<T>(dy[v], d);
    unpack<T>(z[v], f);
    if (ACT != SP24_ACT_NONE) {
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        float2 slope;
        act_and_slope<ACT>(f[n], &slope);
        d[n] = mul2(d[n], slope);
      }
    }
    const uint4 packed = pack<T>(d);
    if (p.dz && r < p.rows && c < p.cols) *reinterpret_cast<uint4*>(static_cast<T*>(p.dz) + r * p.lddz + c) = packed;
    tile[m * kUnits + (u ^ (2 * (m >> 3 & 3) + (m & 1)))] = packed;
    if (p.partial && p.over_rows) {
#pragma unroll
      for (int n = 0; n < 4; ++n) sums[n] = make_float2(sums[n].x + d[n].x, sums[n].y + d[n].y);
    } else if (p.partial) {
      float s = ((d[0].x + d[0].y) + (d[1].x + d[1].y)) + ((d[2].x + d[2].y) + (d[3].x + d[3].y));
#pragma unroll
      for (int i = 1; i < kUnits; i *= 2) s += __shfl_xor_sync(~0u, s, i);
      if (u == 0 && r < p.rows) p.partial[col0 / kWide * p.rows + r] = s;
    }
  }
  if (p.partial && p.over_rows) {
#pragma unroll
    for (int i = kUnits; i < 32; i *= 2)
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        sums[n].x += __shfl_xor_sync(~0u, sums[n].x, i);
        sums[n].y += __shfl_xor_sync(~0u, sums[n].y, i);
      }
    if (lane < kUnits) {
#pragma unroll
      for (int n = 0; n < 4; ++n) *reinterpret_cast<float2*>(&over[warp][8 * u + 2 * n]) = sums[n];
    }
  }
  __syncthreads();
  if (p.dzt) {
    static_assert(kWideThreads / 32 == kUnits, "a warp to a unit: eight columns");
    const int i = lane >> 3, j = (lane & 7) >> 1, b = lane & 1;  // this lane's row of matrix i for ldmatrix
    const int64_t col = col0 + 8 * warp + (lane >> 2);
#pragma unroll
    for (int k = 0; k < kWide / 32; ++k) {
      const int m = 32 * k + 8 * j + 2 * i + b;
      uint32_t x[4];
      ptx::ldmatrix_x4_trans(ptx::smem_u32(&tile[m * kUnits + (warp ^ (2 * (m >> 3 & 3) + (m & 1)))]), x[0], x[1], x[2], x[3]);
      const int64_t r = row0 + 32 * k + 8 * (lane & 3);
      if (col < p.cols && r < p.rows) *reinterpret_cast<uint4*>(static_cast<T*>(p.dzt) + col * p.lddzt + r) = make_uint4(x[0], x[1], x[2], x[3]);
    }
  }
  if (p.partial && p.over_rows && threadIdx.x < kWide) {
    float s = over[0][threadIdx.x];
#pragma unroll
    for (int w = 1; w < kWideThreads / 32; ++w) s += over[w][threadIdx.x];
    if (col0 + threadIdx.x < p.cols) p.partial[row0 / kWide * p.cols + col0 + threadIdx.x] = s;
  }
}

// Any type, size and alignment, element by element through shared memory.
template <typename T, int ACT>
__global__ void __launch_bounds__(256) act_grad_kernel(const ActGradParams p) {
  __shared__ float tile[kTile][kTile + 1];
  wait_for_stream();
  const int64_t col_tiles = (p.cols + kTile - 1) / kTile;
  const int64_t row0 = (int64_t)(blockIdx.x / col_tiles) * kTile, col0 = (int64_t)(blockIdx.x % col_tiles) * kTile;
  const int x = threadIdx.x % kTile, y = threadIdx.x / kTile;
  for (int i = y; i < kTile; i += 256 / kTile) {
    const int64_t r = row0 + i, c = col0 + x;
    float d = 0.f;
    if (r < p.rows && c < p.cols) {
      d = to_float(static_cast<const T*>(p.dy)[r * p.lddy + c]);
      if (ACT != SP24_ACT_NONE) {
        float2 slope;
        act_and_slope<ACT>(both(to_float(static_cast<const T*>(p.z)[r * p.ldz + c])), &slope);
        d *= slope.x;
      }
      if (p.dz) static_cast<T*>(p.dz)[r * p.lddz + c] = round_to<T>(d);
    }
    tile[i][x] = d;
  }
  __syncthreads();
  if (p.dzt)
    for (int i = y; i < kTile; i += 256 / kTile) {
      const int64_t c = col0 + i, r = row0 + x;
      if (r < p.rows && c < p.cols) static_cast<T*>(p.dzt)[c * p.lddzt + r] = round_to<T>(tile[x][i]);
    }
  if (p.partial && threadIdx.x < kTile) {
    float sum = 0.f;
    for (int i = 0; i < kTile; ++i) sum += p.over_rows ? tile[i][threadIdx.x] : tile[threadIdx.x][i];
    const int64_t at = (p.over_rows ? col0 : row0) + threadIdx.x;
    if (p.over_rows && at < p.cols) p.partial[row0 / kTile * p.cols + at] = sum;
    if (!p.over_rows && at < p.rows) p.partial[col0 / kTile * p.rows + at] = sum;
  }
}

// ---- experts ----------------------------------------------------------------------------------------------------------
// Rows [lo, hi) of expert e, as the products take them.
__device__ __forceinline__ void rows_of_expert(const ActGradParams& p, int e, int64_t& lo, int64_t& hi) {
  lo = min(max((int64_t)p.offsets[e], (int64_t)0), p.rows);
  hi = max(lo, min((int64_t)p.offsets[e + 1], p.rows));
}
// The first expert whose rows end behind row r, E if there is none (offsets in order).
__device__ __forceinline__ int expert_of_row(const ActGradParams& p, int64_t r) {
  int lo = 0, hi = p.experts;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (p.offsets[mid + 1] > r) hi = mid;
    else lo = mid + 1;
  }
  return lo;
}

// dz is rounded to the operands' 16 bits, because what reads it are two products of 16-bit tensor-core operands (kept in FP32 it would be TF32 ones at half the rate, over
// twice the bytes): dX and dW are off by the roundings of dz as well as by their own (bf16 8192 rows of 8 experts 4096 x 2048, against FP64: 0.0023, 0.0017 without).
// The sums are of the values before it.
// dz, and the bias's gradient of each expert's rows: tile i of kTile rows has a partial sum of its own for every expert that it meets, in row i + (expert) of
// `partial`, which no other tile and expert share.  16-bit types, rows of whole vectors at 16-byte boundaries.  The tile's values go through shared memory in FP32, where a
// column's sum may end at any row.  Bound by HBM and the arithmetic of the slope: us, device, bf16 8192 x 4096 in 8 experts, GELU 46, SiLU 44, without the sums 35 (floor 31);
// 2048 x 4096 in 64 18.5 (with sums over the lanes of a tile of 128 x 128, and once more from dy and z for each expert of a tile that several share, 50, 45, 37 and 32).
template <typename T, int ACT>
__global__ void __launch_bounds__(256) expert_act_grad_kernel(const ActGradParams p) {
  constexpr int kUnits = kTile / 8, kPasses = kTile * kUnits / 256, kRows = kTile / kPasses;
  __shared__ __align__(16) float tile[kTile][kTile + 4];
  __shared__ float over[4][kTile];
  const int64_t col_tiles = (p.cols + kTile - 1) / kTile;
  const int64_t row0 = (int64_t)(blockIdx.x / col_tiles) * kTile, col0 = (int64_t)(blockIdx.x % col_tiles) * kTile;
  const int u = threadIdx.x % kUnits, m0 = threadIdx.x / kUnits;
  const int64_t c = col0 + 8 * u;
  wait_for_stream();
  uint4 dy[kPasses] = {}, z[kPasses] = {};
#pragma unroll
  for (int v = 0; v < kPasses; ++v)
    if (const int64_t r = row0 + m0 + kRows * v; r < p.rows && c < p.cols) dy[v] = ld_stream(static_cast<const T*>(p.dy) + r * p.lddy + c);
  if (ACT != SP24_ACT_NONE) {
#pragma unroll
    for (int v = 0; v < kPasses; ++v)
      if (const int64_t r = row0 + m0 + kRows * v; r < p.rows && c < p.cols) z[v] = ld_stream(static_cast<const T*>(p.z) + r * p.ldz + c);
  }
#pragma unroll
  for (int v = 0; v < kPasses; ++v) {
    const int m = m0 + kRows * v;
    const int64_t r = row0 + m;
    Pairs<T> d, f;
    unpack<T>(dy[v], d);
    unpack<T>(z[v], f);
    if (ACT != SP24_ACT_NONE) {
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        float2 slope;
        act_and_slope<ACT>(f[n], &slope);
        d[n] = mul2(d[n], slope);
      }
    }
    if (p.dz && r < p.rows && c < p.cols) *reinterpret_cast<uint4*>(static_cast<T*>(p.dz) + r * p.lddz + c) = pack<T>(d);
    if (p.partial) {
      *reinterpret_cast<float4*>(&tile[m][8 * u]) = make_float4(d[0].x, d[0].y, d[1].x, d[1].y);
      *reinterpret_cast<float4*>(&tile[m][8 * u + 4]) = make_float4(d[2].x, d[2].y, d[3].x, d[3].y);
    }
  }
  if (!p.partial) return;
  int e = 0;  // the first expert whose rows end behind row0
  for (int i = 0; i < p.experts; i += 256) e += __syncthreads_count(i + threadIdx.x < p.experts && p.offsets[i + threadIdx.x + 1] <= row0);
  const int64_t end = min(p.rows, row0 + kTile);
  const int x = threadIdx.x % kTile, y = threadIdx.x / kTile;
  for (; e < p.experts; ++e) {
    int64_t lo, hi;
    rows_of_expert(p, e, lo, hi);
    if (lo >= end) break;
    if (hi <= lo) continue;
    const int first = max((int)(max(lo, row0) - row0), y * (kTile / 4)), last = min((int)(min(hi, end) - row0), (y + 1) * (kTile / 4));
    float sum = 0.f;
#pragma unroll 8
    for (int m = first; m < last; ++m) sum += tile[m][x];
    over[y][x] = sum;
    __syncthreads();
    if (y == 0 && col0 + x < p.cols) p.partial[(row0 / kTile + e) * p.cols + col0 + x] = (over[0][x] + over[1][x]) + (over[2][x] + over[3][x]);
    __syncthreads();
  }
}

// The partial sums of the experts' rows for any type, size and alignment: tiles of kTile rows as above.
template <typename T, int ACT>
__global__ void __launch_bounds__(256) expert_sums_kernel(const ActGradParams p) {
  __shared__ float over[4][kTile];
  wait_for_stream();
  const int x = threadIdx.x % kTile, y = threadIdx.x / kTile;
  const int64_t col_tiles = (p.cols + kTile - 1) / kTile, tile = blockIdx.x / col_tiles;
  const int64_t row0 = tile * kTile, end = min(p.rows, row0 + kTile), c = blockIdx.x % col_tiles * kTile + x;
  for (int e = expert_of_row(p, row0); e < p.experts; ++e) {
    int64_t lo, hi;
    rows_of_expert(p, e, lo, hi);
    if (lo >= end) break;
    if (hi <= lo) continue;
    float sum = 0.f;
    if (c < p.cols)
      for (int64_t r = max(lo, row0) + y; r < min(hi, end); r += 4) {
        float d = to_float(static_cast<const T*>(p.dy)[r * p.lddy + c]);
        if (ACT != SP24_ACT_NONE) {
          float2 slope;
          act_and_slope<ACT>(both(to_float(static_cast<const T*>(p.z)[r * p.ldz + c])), &slope);
          d *= slope.x;
        }
        sum += d;
      }
    over[y][x] = sum;
    __syncthreads();
    if (y == 0 && c < p.cols) p.partial[(tile + e) * p.cols + c] = (over[0][x] + over[1][x]) + (over[2][x] + over[3][x]);
    __syncthreads();
  }
}

// An expert's partial sums added up, tile after tile: four tiles side by side, so that a long chain of loads is a quarter as long.
__global__ void __launch_bounds__(256) expert_bias_kernel(const ActGradParams p, float* dbias) {
  __shared__ float over[4][kTile];
  wait_for_stream();
  const int x = threadIdx.x % kTile, y = threadIdx.x / kTile, e = blockIdx.y;
  const int64_t c = (int64_t)blockIdx.x * kTile + x;
  int64_t lo, hi;
  rows_of_expert(p, e, lo, hi);
  float sum = 0.f;
  if (hi > lo && c < p.cols)
    for (int64_t i = lo / kTile + y; i <= (hi - 1) / kTile; i += 4) sum += p.partial[(i + e) * p.cols + c];
  over[y][x] = sum;
  __syncthreads();
  if (y == 0 && c < p.cols) dbias[(int64_t)e * p.cols + c] = (over[0][x] + over[1][x]) + (over[2][x] + over[3][x]);
}

}  // namespace
}  // namespace sp24

using namespace sp24;

extern "C" size_t sp24_act_backward_workspace_bytes(int64_t rows, int64_t cols, int sum_over_rows) {
  if (rows <= 0 || cols <= 0 || rows > kMostColumns || cols > kMostColumns) return 0;
  const int64_t tiles = ((sum_over_rows ? rows : cols) + kTile - 1) / kTile;
  return (size_t)tiles * (size_t)(sum_over_rows ? cols : rows) * sizeof(float);
}

extern "C" sp24_status sp24_act_backward(sp24_dtype t, sp24_act act, int64_t rows, int64_t cols, const void* dy, int64_t lddy, const void* z,
                                         int64_t ldz, void* dz, int64_t lddz, void* dzt, int64_t lddzt, float* dbias, int sum_over_rows,
                                         void* workspace, size_t workspace_bytes, void* stream) {
  SP24_RETURN_IF(!is_float_type(t), SP24_ERR_DTYPE);
  SP24_RETURN_IF(!is_act(act), SP24_ERR_UNSUPPORTED);
  SP24_RETURN_IF(rows < 0 || cols < 0 || rows > kMostColumns || cols > kMostColumns, SP24_ERR_SHAPE);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int64_t sums = sum_over_rows ? cols : rows;
  SP24_RETURN_IF(!aligned(dbias, 4), SP24_ERR_ALIGN);
  if (rows == 0 || cols == 0) {
    if (!dbias || sums == 0) return SP24_OK;
    const sp24_status st = check_arch();
    return st != SP24_OK ? st : cuda_status(cudaMemsetAsync(dbias, 0, (size_t)sums * sizeof(float), s));
  }
  const bool reads_z = act != SP24_ACT_NONE;
  SP24_RETURN_IF(!dy || (reads_z && !z), SP24_ERR_NULL);
  SP24_RETURN_IF(!row_fits(rows, cols, lddy) || (reads_z && !row_fits(rows, cols, ldz)) || (dz && !row_fits(rows, cols, lddz)) ||
                     (dzt && !row_fits(cols, rows, lddzt)),
                 SP24_ERR_STRIDE);
  const size_t es = elem_bytes(t);
  SP24_RETURN_IF(!aligned(dy, es) || (reads_z && !aligned(z, es)) || !aligned(dz, es) || !aligned(dzt, es), SP24_ERR_ALIGN);
  SP24_RETURN_IF(dbias && (!workspace || !aligned16(workspace) || workspace_bytes < sp24_act_backward_workspace_bytes(rows, cols, sum_over_rows)),
                 SP24_ERR_WORKSPACE);
  if (!dz && !dzt && !dbias) return SP24_OK;
  const bool whole = t != SP24_F32 && cols % 8 == 0 && (!dzt || rows % 8 == 0) && whole_rows(dy, rows, lddy, 2, 16) &&
                     (!reads_z || whole_rows(z, rows, ldz, 2, 16)) && whole_rows(dz, rows, lddz, 2, 16) && whole_rows(dzt, cols, lddzt, 2, 16);
  const bool wide = whole && (rows + 127) / 128 * ((cols + 127) / 128) >= 2 * sm_count();
  const int64_t edge = wide ? 2 * kTile : kTile;  // (the workspace has room for the sums of the smaller tiles)
  const int64_t row_tiles = (rows + edge - 1) / edge, col_tiles = (cols + edge - 1) / edge;
  SP24_RETURN_IF(row_tiles * col_tiles > 0x7fffffff, SP24_ERR_SHAPE);
  sp24_status st = check_arch();
  if (st != SP24_OK) return st;
  const ActGradParams p = {rows, cols, dy, z, dz, dzt, dbias ? static_cast<float*>(workspace) : nullptr, lddy, ldz, lddz, lddzt, sum_over_rows != 0};
  const dim3 grid((unsigned)(row_tiles * col_tiles));
  st = with_float_type(t, [&](auto type) {
    using T = typename decltype(type)::type;
    return with_act(act, [&](auto a) {
      if constexpr (sizeof(T) == 2)
        if (whole)
          return launch_overlapped(wide ? act_grad_tile_kernel<T, decltype(a)::value, 2 * kTile> : act_grad_tile_kernel<T, decltype(a)::value, kTile>, grid,
                                   dim3((unsigned)(4 * edge)), 0, s, 1, p);
      return launch_overlapped(act_grad_kernel<T, decltype(a)::value>, grid, dim3(256), 0, s, 1, p);
    });
  });
  if (st != SP24_OK || !dbias) return st;
  return column_sums(static_cast<const float*>(workspace), sum_over_rows ? row_tiles : col_tiles, sums, dbias, s);
}

extern "C" size_t sp24_expert_act_backward_workspace_bytes(int64_t E, int64_t M, int64_t rows) {
  if (E < 1 || E > kMostExperts || M < 1 || M > kMostColumns || rows < 0 || rows > kMostColumns) return 0;
  return (size_t)((rows + kTile - 1) / kTile + E) * (size_t)M * sizeof(float);
}

extern "C" sp24_status sp24_expert_act_backward(sp24_dtype t, sp24_act act, int64_t E, int64_t M, int64_t rows, const void* dy, int64_t lddy,
                                                const void* z, int64_t ldz, const int32_t* offsets, void* dz, int64_t lddz, float* dbias, void* workspace,
                                                size_t workspace_bytes, void* stream) {
  SP24_RETURN_IF(!is_float_type(t), SP24_ERR_DTYPE);
  SP24_RETURN_IF(!is_act(act), SP24_ERR_UNSUPPORTED);
  SP24_RETURN_IF(E < 1 || E > kMostExperts || M < 1 || M > kMostColumns || rows < 0 || rows > kMostColumns, SP24_ERR_SHAPE);
  const bool reads_z = act != SP24_ACT_NONE;
  SP24_RETURN_IF((rows > 0 && (!dy || (reads_z && !z))) || (dbias && !offsets), SP24_ERR_NULL);
  SP24_RETURN_IF(!row_fits(rows, M, lddy) || (reads_z && !row_fits(rows, M, ldz)) || (dz && !row_fits(rows, M, lddz)), SP24_ERR_STRIDE);
  const size_t es = elem_bytes(t);
  SP24_RETURN_IF(!aligned(dy, es) || (reads_z && !aligned(z, es)) || !aligned(dz, es) || !aligned(dbias, 4) || !aligned(offsets, 4), SP24_ERR_ALIGN);
  SP24_RETURN_IF(dbias && (!workspace || !aligned16(workspace) || workspace_bytes < sp24_expert_act_backward_workspace_bytes(E, M, rows)), SP24_ERR_WORKSPACE);
  if (!dbias && (rows == 0 || !dz)) return SP24_OK;
  const int64_t width = M * (int64_t)es;
  const RowsAt result = {dz, rows, width, lddz * (int64_t)es};
  SP24_RETURN_IF(overlap(result, {dy, rows, width, lddy * (int64_t)es}) || (reads_z && overlap(result, {z, rows, width, ldz * (int64_t)es})), SP24_ERR_UNSUPPORTED);
  const bool whole = t != SP24_F32 && M % 8 == 0 && whole_rows(dy, rows, lddy, 2, 16) && (!reads_z || whole_rows(z, rows, ldz, 2, 16)) &&
                     whole_rows(dz, rows, lddz, 2, 16);
  const int64_t row_tiles = (rows + kTile - 1) / kTile, col_tiles = (M + kTile - 1) / kTile;
  SP24_RETURN_IF(row_tiles * col_tiles > 0x7fffffff, SP24_ERR_SHAPE);
  sp24_status st = check_arch();
  SP24_RETURN_IF(st != SP24_OK, st);
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  ActGradParams p = {rows, M, dy, z, dz, nullptr, dbias ? static_cast<float*>(workspace) : nullptr, lddy, ldz, lddz, 0, 1, offsets, (int)E};
  if (rows > 0) {
    const dim3 grid((unsigned)(row_tiles * col_tiles));
    st = with_float_type(t, [&](auto type) {
      using T = typename decltype(type)::type;
      return with_act(act, [&](auto a) {
        constexpr int kAct = decltype(a)::value;
        if constexpr (sizeof(T) == 2)
          if (whole) return launch_overlapped(expert_act_grad_kernel<T, kAct>, grid, dim3(256), 0, s, 1, p);
        ActGradParams q = p;
        q.partial = nullptr;
        sp24_status done = SP24_OK;
        if (dz) done = launch_overlapped(act_grad_kernel<T, kAct>, grid, dim3(256), 0, s, 1, q);
        if (done != SP24_OK || !dbias) return done;
        return launch_overlapped(expert_sums_kernel<T, kAct>, grid, dim3(256), 0, s, 1, p);
      });
    });
    SP24_RETURN_IF(st != SP24_OK || !dbias, st);
  }
  return launch_overlapped(expert_bias_kernel, dim3((unsigned)((M + kTile - 1) / kTile), (unsigned)E), dim3(256), 0, s, 1, p, dbias);
}
