// The order of rows by experts, and the rows' way there and back.
#include "sp24_ptx.cuh"
#include "sp24_rows.cuh"

namespace sp24 {
namespace {

// ---- order ------------------------------------------------------------------------------------------------------
// A stable counting sort.  Each warp has a part of the slots in their order and counts them by experts in shared memory; the counts of a block's warps and then of the
// blocks are added up from the left, and the warp goes over its slots again with the places found (32 at a time, equal ones found by a match over the warp).
// Up to kClusterSlots slots in one launch, of a cluster of up to eight blocks that read one another's counts; the match, about 100 cycles each of an SM's
// memory pipe, is what bounds it then, so more slots go to up to 128 blocks: their counts by a launch before
// (us, device, 131072 slots of 256 experts: 29 by a cluster, 10.5; by 64 blocks 11.1, by 32 13.3; 4096 slots of 64 experts by a cluster 4.5; 256 of 64 2.5).
struct OrderParams {
  int64_t slots, rows;
  int E, align;
  const int32_t* experts;
  int32_t *offsets, *position, *source;
  int32_t* counts;  // [blocks][E], where the counts come by a launch of their own
};
constexpr int64_t kClusterSlots = 8192, kMostOrderBlocks = 128;

__device__ __forceinline__ void slots_of_warp(const OrderParams& p, int block, int blocks, int warp, int warps, int64_t& begin, int64_t& end) {
  const int64_t groups = (p.slots + 31) / 32, per_warp = (groups + (int64_t)blocks * warps - 1) / ((int64_t)blocks * warps);
  begin = ((int64_t)block * warps + warp) * per_warp * 32;
  end = min(p.slots, begin + per_warp * 32);
}
__device__ __forceinline__ int expert_of(const OrderParams& p, int64_t i, int64_t end) {
  const int e = i < end ? p.experts[i] : -1;
  return e >= 0 && e < p.E ? e : -1;
}

// The block's counts, for order_kernel<true> of the same number of blocks and threads.
__global__ void __launch_bounds__(1024) count_kernel(const OrderParams p) {
  extern __shared__ int32_t counts[];
  for (int i = threadIdx.x; i < p.E; i += blockDim.x) counts[i] = 0;
  const int warps = blockDim.x >> 5;
  int64_t begin, end, none;
  slots_of_warp(p, blockIdx.x, gridDim.x, 0, warps, begin, none);
  slots_of_warp(p, blockIdx.x, gridDim.x, warps - 1, warps, none, end);
  __syncthreads();
  wait_for_stream();
  for (int64_t i = begin + threadIdx.x; i < end; i += blockDim.x) {
    const int e = expert_of(p, i, end);
    if (e >= 0) atomicAdd(&counts[e], 1);  // (a sum of ones: any order)
  }
  __syncthreads();
  for (int i = threadIdx.x; i < p.E; i += blockDim.x) p.counts[(int64_t)blockIdx.x * p.E + i] = counts[i];
}

constexpr int kBatch = 4;
template <bool COUNTED>
__global__ void __launch_bounds__(1024) order_kernel(const OrderParams p) {
  extern __shared__ int32_t counts[];  // [warps][E], then [E] of the block, [E] of the experts' first rows, COUNTED: 2 [E] of all blocks
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int rank = COUNTED ? blockIdx.x : (int)ptx::cluster_ctarank(), blocks = gridDim.x;
  int32_t* of_block = counts + warps * p.E;
  int32_t* first = of_block + p.E;
  __shared__ int32_t of_warps[32];
  for (int i = threadIdx.x; i < (warps + 1) * p.E; i += blockDim.x) counts[i] = 0;
  int64_t begin, end;
  slots_of_warp(p, rank, blocks, warp, warps, begin, end);
  __syncthreads();
  wait_for_stream();
  int32_t* mine = counts + warp * p.E;
  // kBatch groups at a time: their loads are all on the way before the first is used
  for (int64_t i = begin; i < end; i += 32 * kBatch) {
    int e[kBatch];
#pragma unroll
    for (int n = 0; n < kBatch; ++n) e[n] = expert_of(p, i + 32 * n + lane, end);
#pragma unroll
    for (int n = 0; n < kBatch; ++n)
      if (e[n] >= 0) atomicAdd(&mine[e[n]], 1);  // (a sum of ones: any order)
  }
  __syncthreads();
  // counts of the warps before, in the place of the warp's; the block's
  for (int e = threadIdx.x; e < p.E; e += blockDim.x) {
    int32_t n = 0;
    for (int w = 0; w < warps; ++w) {
      const int32_t c = counts[w * p.E + e];
      counts[w * p.E + e] = n;
      n += c;
    }
    of_block[e] = n;
  }
  auto cluster_barrier = [&] {  // (cluster of one: the block's own)
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  };
  if (!COUNTED) cluster_barrier();
  // the experts' numbers of slots over all blocks and over the blocks before this one; then their first rows, by a scan
  int32_t total = 0, before = 0;
  const int e = threadIdx.x;  // (E <= 1024: blocks have at least E threads)
  if (COUNTED) {
    // as many threads to an expert as there are, each with every so manieth block; their sums in shared memory
    int32_t* const totals = first + p.E;
    for (int i = threadIdx.x; i < 2 * p.E; i += blockDim.x) totals[i] = 0;
    __syncthreads();
    const int sides = blockDim.x / p.E, side = threadIdx.x / p.E, x = threadIdx.x - side * p.E;
    if (side < sides) {
#pragma unroll 16
      for (int b = side; b < blocks; b += sides) {
        const int32_t c = p.counts[(int64_t)b * p.E + x];
        if (b < rank) before += c;
        total += c;
      }
      atomicAdd(&totals[x], total);
      atomicAdd(&totals[p.E + x], before);
    }
    __syncthreads();
    total = e < p.E ? totals[e] : 0;
    before = e < p.E ? totals[p.E + e] : 0;
  } else if (e < p.E) {
    for (int b = 0; b < blocks; ++b) {
      int32_t c;
      asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(c) : "r"(ptx::map_to_cta(ptx::smem_u32(of_block + e), (uint32_t)b)) : "memory");
      if (b < rank) before += c;
      total += c;
    }
  }
  const int32_t padded = (total + p.align - 1) / p.align * p.align;
  int32_t sum = padded;
#pragma unroll
  for (int i = 1; i < 32; i <<= 1) {
    const int32_t left = __shfl_up_sync(~0u, sum, i);
    if (lane >= i) sum += left;
  }
  if (lane == 31) of_warps[warp] = sum;
  __syncthreads();
  int32_t left = lane < warp ? of_warps[lane] : 0;
  left = __reduce_add_sync(~0u, left);
  const int32_t at = left + sum - padded;
  if (e < p.E) {
    first[e] = at + before;
    if (rank == 0) {
      p.offsets[e] = at;
      if (e == p.E - 1) p.offsets[p.E] = at + padded;
      for (int32_t r = at + total; r < at + padded; ++r) p.source[r] = -1;
    }
  }
  __syncthreads();
  // rows behind the last expert
  int32_t all = lane < warps ? of_warps[lane] : 0;
  all = __reduce_add_sync(~0u, all);
  for (int64_t r = all + (int64_t)rank * blockDim.x + threadIdx.x; r < p.rows; r += (int64_t)blocks * blockDim.x) p.source[r] = -1;
  for (int64_t i = begin; i < end; i += 32 * kBatch) {
    int x[kBatch];
    uint32_t same[kBatch];
#pragma unroll
    for (int n = 0; n < kBatch; ++n) x[n] = expert_of(p, i + 32 * n + lane, end);
#pragma unroll
    for (int n = 0; n < kBatch; ++n) same[n] = __match_any_sync(~0u, x[n]);
#pragma unroll
    for (int n = 0; n < kBatch; ++n) {
      if (i + 32 * n >= end) break;
      int32_t row = -1;
      if (x[n] >= 0) row = first[x[n]] + mine[x[n]] + __popc(same[n] & ((1u << lane) - 1));
      __syncwarp();
      if (x[n] >= 0 && lane == __ffs(same[n]) - 1) mine[x[n]] += __popc(same[n]);
      __syncwarp();
      const int64_t at = i + 32 * n + lane;
      if (at < end) {
        p.position[at] = row;
        if (row >= 0) p.source[row] = (int32_t)at;
      }
    }
  }
  if (!COUNTED) cluster_barrier();  // no block leaves while another may still read its counts
}

// ---- rows -------------------------------------------------------------------------------------------------------
// A block has a token, or several one after the other, its threads the row's vectors of 16 bytes; blocks before those look for rows without a slot and clear them.
// WHOLE: rows are whole vectors at 16-byte boundaries.  Else the vectors lie at the boundaries of the row that is written, and what is read is made of the two
// words that it lies in (load_words).  Bound by HBM: us, device, and of the floor at the copy's rate, e4m3 8192 x 4096 to 8 rows each 51 (91 %); bf16 8192 x 4096, 4
// rows each: gathering 56 (91 %), sums 53 (97 %), the sums' gradient 101 (91 %);
// bf16 8192 x 4095, where every row lies otherwise: 62, 88, 152 (by elements 117, 97, 175).
struct RowsParams {
  int64_t T, K, rows;
  int64_t ld_in, ld_out, ld_y, ld_res;  // elements
  int k;
  int clear_blocks, token_blocks;
  const int32_t *position, *source;
  const void *in, *y, *residual;
  void* out;
  const float* weights;  // gather: scales
  float* sums;           // gather: the rows' scales; the sums' gradient: that of the weights
};

// The first p.clear_blocks blocks.  A warp looks at 32 rows at a time, as far apart as there are warps: rows without a slot come in long runs, behind the last expert.
// (With a block to 256 rows in a row, 1216 rows of 4096 bf16 values, 960 of them empty, took 27 us; 5.5.)
template <bool WHOLE, typename E>
__device__ void clear_rows(const RowsParams& p, float* scale) {
  constexpr int N = kVector<E>;
  const int lane = threadIdx.x & 31;
  const int64_t warps = (int64_t)p.clear_blocks * (blockDim.x >> 5), warp = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  for (int64_t r0 = warp; r0 < p.rows; r0 += 32 * warps) {
    const int64_t r = r0 + lane * warps;
    const bool empty = r < p.rows && p.source[r] < 0;
    if (empty && scale) scale[r] = 0.f;
    uint32_t left = __ballot_sync(~0u, empty);
    while (left) {
      E* row = static_cast<E*>(p.out) + (r0 + (__ffs(left) - 1) * warps) * p.ld_out;
      left &= left - 1;
      const int shift = WHOLE ? 0 : shift_of<E, N>(row);
      for (int c = lane; c * N - shift < p.K; c += 32) store_vector<WHOLE>(row, c, (int)p.K, shift, make_uint4(0, 0, 0, 0));
    }
  }
}

// A token's row is read once (again from the L1 where rows lie between boundaries) and written to its k places.
template <typename E, bool WHOLE>
__global__ void __launch_bounds__(256) gather_kernel(const RowsParams p) {
  constexpr int N = kVector<E>;
  __shared__ int32_t place[kMostChosen];
  wait_for_stream();
  if (blockIdx.x < p.clear_blocks) {
    clear_rows<WHOLE, E>(p, p.sums);
    return;
  }
  const int K = (int)p.K;
  for (int64_t t = blockIdx.x - p.clear_blocks; t < p.T; t += p.token_blocks) {
    __syncthreads();
    if (threadIdx.x < p.k) {
      int32_t r = p.position[t * p.k + threadIdx.x];
      if (r >= p.rows) r = -1;
      place[threadIdx.x] = r;
      if (p.sums && r >= 0) p.sums[r] = p.weights[t];
    }
    __syncthreads();
    const E* row = static_cast<const E*>(p.in) + t * p.ld_in;
    if constexpr (WHOLE) {
      for (int c = threadIdx.x; c * N < K; c += blockDim.x) {
        const uint4 v = reinterpret_cast<const uint4*>(row)[c];
        for (int i = 0; i < p.k; ++i)
          if (place[i] >= 0) store_vector<true>(static_cast<E*>(p.out) + place[i] * p.ld_out, c, K, 0, v);
      }
    } else {
      // (place after place: four of them together took 81 us where this takes 62, bf16 8192 x 4095, 4 rows each)
      for (int i = 0; i < p.k; ++i) {
        if (place[i] < 0) continue;
        E* out = static_cast<E*>(p.out) + place[i] * p.ld_out;
        const int shift = shift_of<E, N>(out);
#pragma unroll 2
        for (int c = threadIdx.x; c * N - shift < K; c += blockDim.x) store_vector<false>(out, c, K, shift, load_vector<false>(row, c, K, shift));
      }
    }
  }
}

// What a vector of a row is made of, and the vector: of FP32 rows between boundaries its four elements (us, 2048 x 4095, 4 rows each: two words and selects 48, 31), else load_words.
template <bool WHOLE, typename T>
using Parts = std::conditional_t<!WHOLE && sizeof(T) == 4, uint4, Words<WHOLE>>;
template <bool WHOLE, typename T>
__device__ __forceinline__ void load_parts(Parts<WHOLE, T>& to, const T* row, int i, int K, int shift) {
  if constexpr (!WHOLE && sizeof(T) == 4) {
    const int e = 4 * i - shift;
    const uint32_t* at = reinterpret_cast<const uint32_t*>(row) + e;
    to.x = (unsigned)e < (unsigned)K ? at[0] : 0u;
    to.y = (unsigned)(e + 1) < (unsigned)K ? at[1] : 0u;
    to.z = (unsigned)(e + 2) < (unsigned)K ? at[2] : 0u;
    to.w = (unsigned)(e + 3) < (unsigned)K ? at[3] : 0u;
  } else {
    load_words<WHOLE>(to, row, i, K, shift);
  }
}
template <bool WHOLE, typename T>
__device__ __forceinline__ uint4 from_parts(const Parts<WHOLE, T>& from, const T* row, int i, int K, int shift) {
  if constexpr (!WHOLE && sizeof(T) == 4) return from;
  else return vector_of<WHOLE>(from, row, i, K, shift);
}

// U vectors of a row and four rows on the way at a time; the sum goes by the slots' order.
template <typename T, bool WHOLE>
__global__ void __launch_bounds__(256, 4) combine_kernel(const RowsParams p) {
  constexpr int kRows = 4, U = WHOLE ? 2 : 1, N = kVector<T>;
  wait_for_stream();
  const int lane = threadIdx.x & 31, K = (int)p.K;
  for (int64_t t = blockIdx.x; t < p.T; t += gridDim.x) {
    int32_t place = lane < p.k ? p.position[t * p.k + lane] : -1;
    if (place >= p.rows) place = -1;
    const float weight = lane < p.k && p.weights ? p.weights[t * p.k + lane] : 1.f;
    T* out = static_cast<T*>(p.out) + t * p.ld_out;
    const int shift = WHOLE ? 0 : shift_of<T, N>(out);
    const T* residual = p.residual ? static_cast<const T*>(p.residual) + t * p.ld_res : nullptr;
    for (int c0 = 0; c0 * N - shift < K; c0 += U * blockDim.x) {
      const int c = c0 + threadIdx.x;
      Parts<WHOLE, T> rest[U] = {};
      if (residual) {
#pragma unroll
        for (int u = 0; u < U; ++u) load_parts<WHOLE, T>(rest[u], residual, c + u * blockDim.x, K, shift);
      }
      Pairs<T> sum[U] = {};
      for (int i0 = 0; i0 < p.k; i0 += kRows) {
        Parts<WHOLE, T> y[kRows][U] = {};
        const T* row[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
          const int32_t r = __shfl_sync(~0u, place, min(i0 + i, 31));
          row[i] = i0 + i < p.k && r >= 0 ? static_cast<const T*>(p.y) + r * p.ld_y : nullptr;
          if (row[i]) {
#pragma unroll
            for (int u = 0; u < U; ++u) load_parts<WHOLE, T>(y[i][u], row[i], c + u * blockDim.x, K, shift);
          }
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
          const float w = __shfl_sync(~0u, weight, min(i0 + i, 31));
          if (!row[i]) continue;
#pragma unroll
          for (int u = 0; u < U; ++u) {
            Pairs<T> x;
            unpack<T>(from_parts<WHOLE, T>(y[i][u], row[i], c + u * blockDim.x, K, shift), x);
#pragma unroll
            for (int n = 0; n < N / 2; ++n) sum[u][n] = fma2(both(w), x[n], sum[u][n]);
          }
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (residual) {
          Pairs<T> x;
          unpack<T>(from_parts<WHOLE, T>(rest[u], residual, c + u * blockDim.x, K, shift), x);
#pragma unroll
          for (int n = 0; n < N / 2; ++n) sum[u][n] = make_float2(sum[u][n].x + x[n].x, sum[u][n].y + x[n].y);
        }
        store_vector<WHOLE>(out, c + u * blockDim.x, K, shift, pack<T>(sum[u]));
      }
    }
  }
}

// in: dout, y, out: dy, sums: dweights.  V vectors of a row and kRows of its k rows on the way at a time; WHOLE: the token's gradient stays in registers while they go by (else the
// vectors of each row lie otherwise).  The k sums meet in shared memory once.
template <typename T, bool WHOLE, int V>
__global__ void __launch_bounds__(256) combine_backward_kernel(const RowsParams p) {
  constexpr int kRows = WHOLE ? 4 : 2, N = kVector<T>;
  static_assert(WHOLE || V == 1, "vectors at the boundaries of each row");
  __shared__ float parts[2][kMostChosen][8];
  wait_for_stream();
  if (blockIdx.x < p.clear_blocks) {
    clear_rows<WHOLE, T>(p, nullptr);
    return;
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, K = (int)p.K, step = V * blockDim.x;
  int turn = 0;
  for (int64_t t = blockIdx.x - p.clear_blocks; t < p.T; t += p.token_blocks, turn ^= 1) {  // (a buffer is written again behind the other one's barrier)
    const T* d_row = static_cast<const T*>(p.in) + t * p.ld_in;
    int32_t place = lane < p.k ? p.position[t * p.k + lane] : -1;
    if (place >= p.rows) place = -1;
    const float weight = lane < p.k ? p.weights[t * p.k + lane] : 0.f;
    for (int c0 = 0; c0 * N - (WHOLE ? 0 : N - 1) < K; c0 += step) {
      const int c = c0 + threadIdx.x;
      Parts<WHOLE, T> d[WHOLE ? V : kRows] = {};
      if (WHOLE) {
#pragma unroll
        for (int v = 0; v < V; ++v) load_parts<WHOLE, T>(d[v], d_row, c + v * blockDim.x, K, 0);
      }
      for (int i0 = 0; i0 < p.k; i0 += kRows) {
        Parts<WHOLE, T> y[kRows][V] = {};
        int32_t r[kRows];
        int shift[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
          r[i] = __shfl_sync(~0u, place, min(i0 + i, 31));
          if (i0 + i >= p.k) r[i] = -1;
          shift[i] = 0;
          if (r[i] >= 0) {
            if (!WHOLE) {
              shift[i] = shift_of<T, N>(static_cast<T*>(p.out) + r[i] * p.ld_out);
              load_parts<WHOLE, T>(d[i], d_row, c, K, shift[i]);
            }
#pragma unroll
            for (int v = 0; v < V; ++v) load_parts<WHOLE, T>(y[i][v], static_cast<const T*>(p.y) + r[i] * p.ld_y, c + v * blockDim.x, K, shift[i]);
          }
        }
        float dot[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
          dot[i] = 0.f;
          const float w = __shfl_sync(~0u, weight, min(i0 + i, 31));
          if (r[i] >= 0) {
            const T* y_row = static_cast<const T*>(p.y) + r[i] * p.ld_y;
            T* out = static_cast<T*>(p.out) + r[i] * p.ld_out;
#pragma unroll
            for (int v = 0; v < V; ++v) {
              Pairs<T> a, b;
              unpack<T>(from_parts<WHOLE, T>(d[WHOLE ? v : i], d_row, c + v * blockDim.x, K, shift[i]), a);
              unpack<T>(from_parts<WHOLE, T>(y[i][v], y_row, c + v * blockDim.x, K, shift[i]), b);
#pragma unroll
              for (int n = 0; n < N / 2; ++n) {
                dot[i] = fmaf(a[n].x, b[n].x, dot[i]);
                dot[i] = fmaf(a[n].y, b[n].y, dot[i]);
                a[n] = mul2(a[n], both(w));
              }
              store_vector<WHOLE>(out, c + v * blockDim.x, K, shift[i], pack<T>(a));
            }
          }
        }
#pragma unroll
        for (int s = 16; s > 0; s >>= 1)
#pragma unroll
          for (int i = 0; i < kRows; ++i) dot[i] += __shfl_xor_sync(~0u, dot[i], s);
        if (lane == 0) {
#pragma unroll
          for (int i = 0; i < kRows; ++i)
            if (i0 + i < p.k) {
              float& part = parts[turn][i0 + i][warp];
              part = c0 ? part + dot[i] : dot[i];
            }
        }
      }
    }
    __syncthreads();
    if (threadIdx.x < p.k) {
      float sum = parts[turn][threadIdx.x][0];
      for (int w = 1; w < warps; ++w) sum += parts[turn][threadIdx.x][w];
      p.sums[t * p.k + threadIdx.x] = sum;
    }
  }
}

bool code_or_float(sp24_dtype t) { return is_float_type(t) || is_code_type(t) || t == SP24_I32; }

// whether rows of K elements of `es` bytes are whole 16-byte vectors at 16-byte boundaries
bool whole_vectors(int es, int64_t K, std::initializer_list<const void*> at, std::initializer_list<int64_t> lds) {
  bool ok = K * es % 16 == 0;
  for (const void* a : at) ok = ok && aligned16(a);
  for (const int64_t ld : lds) ok = ok && ld * es % 16 == 0;
  return ok;
}

// threads to a row of n vectors: whole warps, at most 256, as many rounds of them as 256 would take
unsigned row_threads(int64_t n) {
  const int64_t rounds = (n + 255) / 256;
  return (unsigned)(((n + rounds - 1) / rounds + 31) / 32 * 32);
}
unsigned token_blocks(int64_t T) {
  const int64_t most = (int64_t)sm_count() * 32;
  return (unsigned)(T < most ? T : most);
}
// blocks that look for rows to clear: a warp to four rows, at most two blocks to an SM
unsigned clearing_blocks(int64_t rows, unsigned threads) {
  const int64_t warps = threads / 32, n = (rows + 4 * warps - 1) / (4 * warps), most = 2 * (int64_t)sm_count();
  return (unsigned)(n < most ? n : most);
}

}  // namespace
}  // namespace sp24

using namespace sp24;

extern "C" int64_t sp24_expert_rows(int64_t slots, int64_t E, int64_t align) {
  if (slots < 0 || E < 1 || align < 1 || slots > (int64_t(1) << 31)) return 0;
  return (slots + (align - 1) * (E < slots ? E : slots) + align - 1) / align * align;
}

extern "C" size_t sp24_expert_order_workspace_bytes(int64_t slots, int64_t E) {
  if (slots <= kClusterSlots || E < 1 || E > kMostExperts) return 0;
  return (size_t)(kMostOrderBlocks * E * 4);
}

extern "C" sp24_status sp24_expert_order(int64_t slots, int64_t E, int64_t align, const int32_t* experts, int32_t* offsets, int32_t* position,
                                         int32_t* source, void* workspace, size_t workspace_bytes, void* stream) {
  SP24_RETURN_IF(slots < 0 || E < 1 || E > kMostExperts || align < 1 || align > 256, SP24_ERR_SHAPE);
  const int64_t rows = sp24_expert_rows(slots, E, align);
  SP24_RETURN_IF(slots >= int64_t(1) << 31 || rows >= int64_t(1) << 31, SP24_ERR_SHAPE);
  SP24_RETURN_IF(offsets == nullptr || (slots > 0 && (experts == nullptr || position == nullptr || source == nullptr)), SP24_ERR_NULL);
  SP24_RETURN_IF(!aligned(experts, 4) || !aligned(offsets, 4) || !aligned(position, 4) || !aligned(source, 4), SP24_ERR_ALIGN);
  const bool counted = slots > kClusterSlots;
  SP24_RETURN_IF(counted && (workspace == nullptr || !aligned16(workspace) || workspace_bytes < sp24_expert_order_workspace_bytes(slots, E)), SP24_ERR_WORKSPACE);
  const sp24_status arch = check_arch();
  SP24_RETURN_IF(arch != SP24_OK, arch);
  OrderParams p = {slots, rows, (int)E, (int)align, experts, offsets, position, source, static_cast<int32_t*>(workspace)};
  // a block to 1024 slots, in a cluster to 512 and eight at most; threads: one to an expert at least, and where there are many experts as many as there can
  // be, to add the blocks' counts up (us, 1024 threads and 512: 131072 slots of 256 experts 10.5, 11.1; 16384 of 64 7.6, 6.2)
  int64_t blocks = 1;
  if (counted) blocks = slots / 1024 < kMostOrderBlocks ? slots / 1024 : kMostOrderBlocks;
  else
    while (blocks < 8 && blocks * 512 < slots) blocks *= 2;
  int64_t threads = (slots + blocks * 32 - 1) / (blocks * 32) * 32;
  if (threads < (E + 31) / 32 * 32) threads = (E + 31) / 32 * 32;
  if (threads > 1024) threads = 1024;
  if (counted) threads = E > 128 ? 1024 : 512;
  const size_t smem = (size_t)((threads / 32 + (counted ? 4 : 2)) * E * 4);
  const auto kernel = counted ? order_kernel<true> : order_kernel<false>;
  static std::atomic<bool> allowed[64];  // the shared-memory opt-in, per device
  int dev = 0;
  SP24_CUDA_CHECK(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64 || !allowed[dev].load(std::memory_order_acquire)) {
    SP24_CUDA_CHECK(cudaFuncSetAttribute(order_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, 36 * kMostExperts * 4));
    SP24_CUDA_CHECK(cudaFuncSetAttribute(order_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, 34 * kMostExperts * 4));
    if (dev >= 0 && dev < 64) allowed[dev].store(true, std::memory_order_release);
  }
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (counted) {
    const sp24_status st = launch_overlapped(count_kernel, dim3((unsigned)blocks), dim3((unsigned)threads), (size_t)(E * 4), s, 1, p);
    SP24_RETURN_IF(st != SP24_OK, st);
  }
  return launch_overlapped(kernel, dim3((unsigned)blocks), dim3((unsigned)threads), smem, s, counted ? 1u : (unsigned)blocks, p);
}

extern "C" sp24_status sp24_expert_gather(sp24_dtype t, int64_t T, int64_t K, const void* x, int64_t ldx, const float* scale, int k,
                                          const int32_t* position, int64_t rows, const int32_t* source, void* out, int64_t ldo, float* out_scale,
                                          void* stream) {
  SP24_RETURN_IF(!code_or_float(t), SP24_ERR_DTYPE);
  SP24_RETURN_IF(T < 0 || K < 1 || K > kMostColumns || rows < 0 || rows >= int64_t(1) << 31 || k < 1 || k > kMostChosen, SP24_ERR_SHAPE);
  if (rows == 0) return SP24_OK;
  SP24_RETURN_IF((T > 0 && (x == nullptr || position == nullptr)) || source == nullptr || out == nullptr || (scale != nullptr) != (out_scale != nullptr),
                 SP24_ERR_NULL);
  SP24_RETURN_IF(!row_fits(T, K, ldx) || !row_fits(rows, K, ldo), SP24_ERR_STRIDE);
  const int es = elem_bytes(t);
  SP24_RETURN_IF(!aligned(x, es) || !aligned(out, es) || !aligned(scale, 4) || !aligned(out_scale, 4) || !aligned(position, 4) || !aligned(source, 4),
                 SP24_ERR_ALIGN);
  const RowsAt result = {out, rows, K * es, ldo * es};
  SP24_RETURN_IF(overlap(result, {x, T, K * es, ldx * es}), SP24_ERR_UNSUPPORTED);
  const sp24_status arch = check_arch();
  SP24_RETURN_IF(arch != SP24_OK, arch);
  RowsParams p = {};
  p.T = T; p.K = K; p.rows = rows; p.k = k;
  p.ld_in = ldx; p.ld_out = ldo;
  p.in = x; p.out = out;
  p.position = position; p.source = source; p.weights = scale; p.sums = out_scale;
  const bool whole = whole_vectors(es, K, {x, out}, {ldx, ldo});
  const unsigned threads = row_threads(row_vectors(K, es, whole));
  p.token_blocks = (int)token_blocks(T);
  p.clear_blocks = (int)clearing_blocks(rows, threads);
  auto run = [&](auto element) {
    using E = decltype(element);
    return launch_overlapped(whole ? gather_kernel<E, true> : gather_kernel<E, false>, dim3(p.token_blocks + p.clear_blocks), dim3(threads), 0,
                             static_cast<cudaStream_t>(stream), 1, p);
  };
  if (es == 4) return run(uint32_t{});
  if (es == 2) return run(uint16_t{});
  return run(uint8_t{});
}

extern "C" sp24_status sp24_expert_combine(sp24_dtype t, int64_t T, int64_t K, int64_t rows, const void* y, int64_t ldy, int k,
                                           const int32_t* position, const float* weights, const void* residual, int64_t ldr, void* out, int64_t ldo,
                                           void* stream) {
  SP24_RETURN_IF(!is_float_type(t), SP24_ERR_DTYPE);
  SP24_RETURN_IF(T < 0 || K < 1 || K > kMostColumns || rows < 0 || rows >= int64_t(1) << 31 || k < 1 || k > kMostChosen, SP24_ERR_SHAPE);
  if (T == 0) return SP24_OK;
  SP24_RETURN_IF((rows > 0 && y == nullptr) || position == nullptr || out == nullptr, SP24_ERR_NULL);
  SP24_RETURN_IF(!row_fits(rows, K, ldy) || !row_fits(T, K, ldo) || (residual && !row_fits(T, K, ldr)), SP24_ERR_STRIDE);
  SP24_RETURN_IF(out == residual && T > 1 && ldo != ldr, SP24_ERR_STRIDE);
  const int es = elem_bytes(t);
  SP24_RETURN_IF(!aligned(y, es) || !aligned(out, es) || !aligned(residual, es) || !aligned(weights, 4) || !aligned(position, 4), SP24_ERR_ALIGN);
  const RowsAt result = {out, T, K * es, ldo * es};
  SP24_RETURN_IF(overlap(result, {y, rows, K * es, ldy * es}) || (residual != out && overlap(result, {residual, T, K * es, ldr * es})), SP24_ERR_UNSUPPORTED);
  const sp24_status arch = check_arch();
  SP24_RETURN_IF(arch != SP24_OK, arch);
  RowsParams p = {};
  p.T = T; p.K = K; p.rows = rows; p.k = k;
  p.ld_y = ldy; p.ld_out = ldo; p.ld_res = ldr;
  p.y = y; p.residual = residual; p.out = out;
  p.position = position; p.weights = weights;
  const bool whole = whole_vectors(es, K, {y, out, residual}, {ldy, ldo, residual ? ldr : 0});
  return with_float_type(t, [&](auto type) {
    using Type = typename decltype(type)::type;
    const int64_t n = row_vectors(K, es, whole);  // (whole vectors: half as many threads with two each, more tokens to an SM)
    return launch_overlapped(whole ? combine_kernel<Type, true> : combine_kernel<Type, false>, dim3(token_blocks(T)), dim3(row_threads(whole ? (n + 1) / 2 : n)), 0,
                             static_cast<cudaStream_t>(stream), 1, p);
  });
}

extern "C" sp24_status sp24_expert_combine_backward(sp24_dtype t, int64_t T, int64_t K, int64_t rows, const void* dout, int64_t lddo, const void* y,
                                                    int64_t ldy, int k, const int32_t* position, const int32_t* source, const float* weights,
                                                    void* dy, int64_t lddy, float* dweights, void* stream) {
  SP24_RETURN_IF(!is_float_type(t), SP24_ERR_DTYPE);
  SP24_RETURN_IF(T < 0 || K < 1 || K > kMostColumns || rows < 0 || rows >= int64_t(1) << 31 || k < 1 || k > kMostChosen, SP24_ERR_SHAPE);
  if (T == 0 && rows == 0) return SP24_OK;
  SP24_RETURN_IF((T > 0 && (dout == nullptr || position == nullptr || weights == nullptr || dweights == nullptr)) ||
                     (rows > 0 && (y == nullptr || source == nullptr || dy == nullptr)), SP24_ERR_NULL);
  SP24_RETURN_IF(!row_fits(T, K, lddo) || !row_fits(rows, K, ldy) || !row_fits(rows, K, lddy), SP24_ERR_STRIDE);
  SP24_RETURN_IF(dy == y && rows > 1 && ldy != lddy, SP24_ERR_STRIDE);
  const int es = elem_bytes(t);
  SP24_RETURN_IF(!aligned(dout, es) || !aligned(y, es) || !aligned(dy, es) || !aligned(weights, 4) || !aligned(dweights, 4) || !aligned(position, 4) ||
                     !aligned(source, 4), SP24_ERR_ALIGN);
  const RowsAt result = {dy, rows, K * es, lddy * es};
  SP24_RETURN_IF(overlap(result, {dout, T, K * es, lddo * es}) || (y != dy && overlap(result, {y, rows, K * es, ldy * es})), SP24_ERR_UNSUPPORTED);
  const sp24_status arch = check_arch();
  SP24_RETURN_IF(arch != SP24_OK, arch);
  RowsParams p = {};
  p.T = T; p.K = K; p.rows = rows; p.k = k;
  p.ld_in = lddo; p.ld_y = ldy; p.ld_out = lddy;
  p.in = dout; p.y = y; p.out = dy;
  p.position = position; p.source = source; p.weights = weights; p.sums = dweights;
  const bool whole = whole_vectors(es, K, {dout, y, dy}, {lddo, ldy, lddy});
  return with_float_type(t, [&](auto type) {
    using Type = typename decltype(type)::type;
    const int64_t n = row_vectors(K, es, whole);
    const unsigned threads = row_threads(n);
    p.token_blocks = (int)token_blocks(T);
    p.clear_blocks = (int)clearing_blocks(rows, threads);
    const auto kernel = !whole ? combine_backward_kernel<Type, false, 1> : n <= threads ? combine_backward_kernel<Type, true, 1> : combine_backward_kernel<Type, true, 2>;
    return launch_overlapped(kernel, dim3(p.token_blocks + p.clear_blocks), dim3(threads), 0, static_cast<cudaStream_t>(stream), 1, p);
  });
}
