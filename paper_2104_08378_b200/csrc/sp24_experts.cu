// The order of rows by experts, and the rows' way there and back.
#include "sp24_ptx.cuh"
#include "sp24_rows.cuh"

namespace sp24 {
namespace {

constexpr int kMostExperts = 1024, kMostChosen = 32;

// ---- order ------------------------------------------------------------------------------------------------------
// A stable counting sort in one launch: a cluster of up to eight blocks, each with a part of the slots in their order, each warp with a part of
// the block's.  A warp counts its slots by experts in shared memory (32 slots at a time, equal ones found by a match over the warp); the
// counts of a block and then of the cluster are added up from the left, and the warp goes over its slots again with the places found.
struct OrderParams {
  int64_t slots, rows;
  int E, align;
  const int32_t* experts;
  int32_t *offsets, *position, *source;
};

__global__ void __launch_bounds__(1024) order_kernel(const OrderParams p) {
  extern __shared__ int32_t counts[];  // [warps][E], then [E] of the block, [E] of the experts' first rows
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const int rank = (int)ptx::cluster_ctarank(), blocks = gridDim.x;
  int32_t* of_block = counts + warps * p.E;
  int32_t* first = of_block + p.E;
  __shared__ int32_t of_warps[32];
  for (int i = threadIdx.x; i < (warps + 1) * p.E; i += blockDim.x) counts[i] = 0;
  // this warp's slots: whole groups of 32
  const int64_t groups = (p.slots + 31) / 32, per_warp = (groups + (int64_t)blocks * warps - 1) / ((int64_t)blocks * warps);
  const int64_t begin = ((int64_t)rank * warps + warp) * per_warp * 32, end = min(p.slots, begin + per_warp * 32);
  __syncthreads();
  wait_for_stream();
  int32_t* mine = counts + warp * p.E;
  auto expert_of = [&](int64_t i) -> int {
    const int e = i < end ? p.experts[i] : -1;
    return e >= 0 && e < p.E ? e : -1;
  };
  for (int64_t i = begin; i < end; i += 32) {
    const int e = expert_of(i + lane);
    const uint32_t same = __match_any_sync(~0u, e);
    if (e >= 0 && lane == __ffs(same) - 1) mine[e] += __popc(same);
    __syncwarp();
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
  // (cluster of one: a barrier of the block's own)
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  // the experts' numbers of slots over all blocks and over the blocks before this one; then their first rows, by a scan
  int32_t total = 0, before = 0;
  const int e = threadIdx.x;  // (E <= 1024: blocks have at least E threads)
  if (e < p.E) {
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
  for (int64_t i = begin; i < end; i += 32) {
    const int x = expert_of(i + lane);
    const uint32_t same = __match_any_sync(~0u, x);
    int32_t row = -1;
    if (x >= 0) row = first[x] + mine[x] + __popc(same & ((1u << lane) - 1));
    __syncwarp();
    if (x >= 0 && lane == __ffs(same) - 1) mine[x] += __popc(same);
    __syncwarp();
    if (i + lane < end) {
      p.position[i + lane] = row;
      if (row >= 0) p.source[row] = (int32_t)(i + lane);
    }
  }
  // no block leaves while another may still read its counts
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// ---- rows -------------------------------------------------------------------------------------------------------
// A block has a token (or several one after the other), its threads the vectors of the row, at most kAhead of them in registers at a time; the
// blocks behind those look for rows without a slot and clear them.  A vector is 16 bytes, or one element of the type where rows are not made of
// whole ones at 16-byte boundaries.
struct RowsParams {
  int64_t T, K, rows;        // K in vectors
  int64_t ld_in, ld_out, ld_y, ld_res;  // bytes
  int k;
  int token_blocks;
  const int32_t *position, *source;
  const uint8_t *in, *y, *residual;
  uint8_t* out;
  const float* weights;  // gather: scales
  float* sums;           // gather: the rows' scales
};

template <typename W>
__device__ __forceinline__ W zero_vector() {
  if constexpr (sizeof(W) == 16) return make_uint4(0, 0, 0, 0);
  else return W(0);
}

template <typename W>
__device__ void clear_rows(const RowsParams& p, int64_t ld, uint8_t* out, float* scale) {
  const int64_t blocks = gridDim.x - p.token_blocks;
  for (int64_t r0 = (int64_t)(blockIdx.x - p.token_blocks) * blockDim.x; r0 < p.rows; r0 += blocks * blockDim.x) {
    const int64_t r = r0 + threadIdx.x;
    const bool empty = r < p.rows && p.source[r] < 0;
    if (empty && scale) scale[r] = 0.f;
    __shared__ int32_t list[1024];
    __shared__ int count;
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    if (empty) list[atomicAdd(&count, 1)] = threadIdx.x;  // (in any order: they all become zeros)
    __syncthreads();
    const int n = count;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    for (int i = warp; i < n; i += warps) {
      W* row = reinterpret_cast<W*>(out + (r0 + list[i]) * ld);
      for (int64_t c = lane; c < p.K; c += 32) row[c] = zero_vector<W>();
    }
    __syncthreads();
  }
}

// A token's row is read once and written to its k places.
template <typename W>
__global__ void __launch_bounds__(256) gather_kernel(const RowsParams p) {
  __shared__ int32_t place[kMostChosen];
  wait_for_stream();
  if (blockIdx.x >= p.token_blocks) {
    clear_rows<W>(p, p.ld_out, p.out, p.sums);
    return;
  }
  for (int64_t t = blockIdx.x; t < p.T; t += p.token_blocks) {
    __syncthreads();
    if (threadIdx.x < p.k) {
      int32_t r = p.position[t * p.k + threadIdx.x];
      if (r >= p.rows) r = -1;
      place[threadIdx.x] = r;
      if (p.sums && r >= 0) p.sums[r] = p.weights[t];
    }
    __syncthreads();
    const W* row = reinterpret_cast<const W*>(p.in + t * p.ld_in);
    for (int64_t c = threadIdx.x; c < p.K; c += blockDim.x) {
      const W v = row[c];
      for (int i = 0; i < p.k; ++i)
        if (place[i] >= 0) reinterpret_cast<W*>(p.out + (int64_t)place[i] * p.ld_out)[c] = v;
    }
  }
}

// Values of a vector as FP32 and back
template <typename T, typename W>
struct Values {
  static constexpr int N = sizeof(W) / sizeof(T);
  float v[N];
  __device__ __forceinline__ void load(const W* at) {
    if constexpr (sizeof(W) == 16) {
      Pairs<T> f;
      unpack<T>(*reinterpret_cast<const uint4*>(at), f);
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        v[2 * i] = f[i].x;
        v[2 * i + 1] = f[i].y;
      }
    } else {
      v[0] = to_float(*reinterpret_cast<const T*>(at));
    }
  }
  __device__ __forceinline__ void store(W* at) const {
    if constexpr (sizeof(W) == 16) {
      Pairs<T> f;
#pragma unroll
      for (int i = 0; i < N / 2; ++i) f[i] = make_float2(v[2 * i], v[2 * i + 1]);
      *reinterpret_cast<uint4*>(at) = pack<T>(f);
    } else {
      *reinterpret_cast<T*>(at) = round_to<T>(v[0]);
    }
  }
};

template <typename T, typename W>
__global__ void __launch_bounds__(256) combine_kernel(const RowsParams p) {
  __shared__ int32_t place[kMostChosen];
  __shared__ float weight[kMostChosen];
  wait_for_stream();
  for (int64_t t = blockIdx.x; t < p.T; t += gridDim.x) {
    __syncthreads();
    if (threadIdx.x < p.k) {
      const int32_t r = p.position[t * p.k + threadIdx.x];
      place[threadIdx.x] = r < p.rows ? r : -1;
      weight[threadIdx.x] = p.weights ? p.weights[t * p.k + threadIdx.x] : 1.f;
    }
    __syncthreads();
    for (int64_t c = threadIdx.x; c < p.K; c += blockDim.x) {
      Values<T, W> sum, x;
#pragma unroll
      for (int n = 0; n < sum.N; ++n) sum.v[n] = 0.f;
      for (int i = 0; i < p.k; ++i) {
        if (place[i] < 0) continue;
        x.load(reinterpret_cast<const W*>(p.y + (int64_t)place[i] * p.ld_y) + c);
#pragma unroll
        for (int n = 0; n < sum.N; ++n) sum.v[n] = fmaf(weight[i], x.v[n], sum.v[n]);
      }
      if (p.residual) {
        x.load(reinterpret_cast<const W*>(p.residual + t * p.ld_res) + c);
#pragma unroll
        for (int n = 0; n < sum.N; ++n) sum.v[n] += x.v[n];
      }
      sum.store(reinterpret_cast<W*>(p.out + t * p.ld_out) + c);
    }
  }
}

// in: dout, y, out: dy, sums: dweights
template <typename T, typename W>
__global__ void __launch_bounds__(256) combine_backward_kernel(const RowsParams p) {
  __shared__ float parts[2][8];
  wait_for_stream();
  if (blockIdx.x >= p.token_blocks) {
    clear_rows<W>(p, p.ld_out, p.out, nullptr);
    return;
  }
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  int turn = 0;
  for (int64_t t = blockIdx.x; t < p.T; t += p.token_blocks) {
    const W* d_row = reinterpret_cast<const W*>(p.in + t * p.ld_in);
    for (int i = 0; i < p.k; ++i) {
      int32_t r = p.position[t * p.k + i];
      if (r >= p.rows) r = -1;
      float dot = 0.f;
      if (r >= 0) {
        const float w = p.weights[t * p.k + i];
        const W* y_row = reinterpret_cast<const W*>(p.y + (int64_t)r * p.ld_y);
        W* out = reinterpret_cast<W*>(p.out + (int64_t)r * p.ld_out);
        for (int64_t c = threadIdx.x; c < p.K; c += blockDim.x) {
          Values<T, W> d, y;
          d.load(d_row + c);
          y.load(y_row + c);
#pragma unroll
          for (int n = 0; n < d.N; ++n) {
            dot = fmaf(d.v[n], y.v[n], dot);
            d.v[n] *= w;
          }
          d.store(out + c);
        }
      }
#pragma unroll
      for (int s = 16; s > 0; s >>= 1) dot += __shfl_xor_sync(~0u, dot, s);
      if (lane == 0) parts[turn][warp] = dot;
      __syncthreads();
      if (threadIdx.x == 0) {
        float sum = parts[turn][0];
        for (int w = 1; w < warps; ++w) sum += parts[turn][w];
        p.sums[t * p.k + i] = sum;
      }
      turn ^= 1;  // (a buffer is written again behind the other one's barrier)
    }
  }
}

// ---- the bias's gradient ------------------------------------------------------------------------------------------
// Sums over an expert's rows in parts of kBiasRows, then over the parts; an expert's parts begin where those of the experts before end at the latest.
constexpr int kBiasRows = 256, kBiasColumns = 64;
struct BiasParams {
  int64_t rows, M, lddy, ldz;
  int E;
  const void *dy, *z;
  const int32_t* offsets;
  float *partial, *dbias;
};
// rows [lo, hi) of expert e, as the products take them
__device__ __forceinline__ void rows_of_expert(const int32_t* offsets, int64_t rows, int e, int64_t& lo, int64_t& hi) {
  lo = min(max((int64_t)offsets[e], (int64_t)0), rows);
  hi = max(lo, min((int64_t)offsets[e + 1], rows));
}

// Block (column tile, part): the part's expert and rows by a search over the offsets.  Parts of expert e are number offsets[e] / kBiasRows + e and on.
template <typename T, int ACT>
__global__ void __launch_bounds__(256) bias_parts_kernel(const BiasParams p) {
  __shared__ float over[4][kBiasColumns];
  wait_for_stream();
  int e = 0, high = p.E - 1;  // the last expert whose first part is not behind this one
  while (e < high) {
    const int mid = (e + high + 1) / 2;
    int64_t lo, hi;
    rows_of_expert(p.offsets, p.rows, mid, lo, hi);
    if (lo / kBiasRows + mid <= blockIdx.y) e = mid;
    else high = mid - 1;
  }
  int64_t lo, hi;
  rows_of_expert(p.offsets, p.rows, e, lo, hi);
  const int64_t begin = lo + ((int64_t)blockIdx.y - (lo / kBiasRows + e)) * kBiasRows, end = min(hi, begin + kBiasRows);
  const int x = threadIdx.x % kBiasColumns, y = threadIdx.x / kBiasColumns;
  const int64_t c = (int64_t)blockIdx.x * kBiasColumns + x;
  float sum = 0.f;
  if (c < p.M && begin >= lo) {
    for (int64_t r = begin + y; r < end; r += 4) {
      float d = to_float(static_cast<const T*>(p.dy)[r * p.lddy + c]);
      if (ACT != SP24_ACT_NONE) {
        float2 slope;
        act_and_slope<ACT>(both(to_float(static_cast<const T*>(p.z)[r * p.ldz + c])), &slope);
        d *= slope.x;
      }
      sum += d;
    }
  }
  over[y][x] = sum;
  __syncthreads();
  if (y == 0 && c < p.M) p.partial[(int64_t)blockIdx.y * p.M + c] = (over[0][x] + over[1][x]) + (over[2][x] + over[3][x]);
}

__global__ void __launch_bounds__(256) bias_sums_kernel(const BiasParams p) {
  wait_for_stream();
  const int64_t c = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  const int e = blockIdx.y;
  if (c >= p.M) return;
  int64_t lo, hi;
  rows_of_expert(p.offsets, p.rows, e, lo, hi);
  const int64_t first = lo / kBiasRows + e, parts = (hi - lo + kBiasRows - 1) / kBiasRows;
  float sum = 0.f;
  for (int64_t i = 0; i < parts; ++i) sum += p.partial[(first + i) * p.M + c];
  p.dbias[(int64_t)e * p.M + c] = sum;
}

bool code_or_float(sp24_dtype t) { return is_float_type(t) || is_code_type(t) || t == SP24_I32; }

// whether rows of K elements of `es` bytes are whole 16-byte vectors at 16-byte boundaries
bool whole_vectors(int es, int64_t K, std::initializer_list<const void*> at, std::initializer_list<int64_t> lds) {
  bool ok = K * es % 16 == 0;
  for (const void* a : at) ok = ok && aligned16(a);
  for (const int64_t ld : lds) ok = ok && ld * es % 16 == 0;
  return ok;
}

// threads to a row of n vectors: whole warps, at most 256
unsigned row_threads(int64_t n) { return (unsigned)(n >= 256 ? 256 : (n + 31) / 32 * 32); }
unsigned token_blocks(int64_t T) {
  const int64_t most = (int64_t)sm_count() * 32;
  return (unsigned)(T < most ? T : most);
}
// blocks that look for rows to clear
unsigned clearing_blocks(int64_t rows, unsigned threads) {
  const int64_t n = (rows + threads - 1) / threads, most = sm_count();
  return (unsigned)(n < most ? n : most);
}

}  // namespace
}  // namespace sp24

using namespace sp24;

extern "C" int64_t sp24_expert_rows(int64_t slots, int64_t E, int64_t align) {
  if (slots < 0 || E < 1 || align < 1 || slots > (int64_t(1) << 31)) return 0;
  return (slots + (align - 1) * (E < slots ? E : slots) + align - 1) / align * align;
}

extern "C" sp24_status sp24_expert_order(int64_t slots, int64_t E, int64_t align, const int32_t* experts, int32_t* offsets, int32_t* position,
                                         int32_t* source, void* stream) {
  SP24_RETURN_IF(slots < 0 || E < 1 || E > kMostExperts || align < 1 || align > 256, SP24_ERR_SHAPE);
  const int64_t rows = sp24_expert_rows(slots, E, align);
  SP24_RETURN_IF(slots >= int64_t(1) << 31 || rows >= int64_t(1) << 31, SP24_ERR_SHAPE);
  SP24_RETURN_IF(offsets == nullptr || (slots > 0 && (experts == nullptr || position == nullptr || source == nullptr)), SP24_ERR_NULL);
  SP24_RETURN_IF(!aligned(experts, 4) || !aligned(offsets, 4) || !aligned(position, 4) || !aligned(source, 4), SP24_ERR_ALIGN);
  const sp24_status arch = check_arch();
  SP24_RETURN_IF(arch != SP24_OK, arch);
  OrderParams p = {slots, rows, (int)E, (int)align, experts, offsets, position, source};
  // threads: one to an expert at least; a block to 2048 slots, eight at most
  int64_t blocks = 1;
  while (blocks < 8 && blocks * 2048 < slots) blocks *= 2;
  int64_t threads = (slots + blocks * 32 - 1) / (blocks * 32) * 32;
  if (threads < (E + 31) / 32 * 32) threads = (E + 31) / 32 * 32;
  if (threads > 1024) threads = 1024;
  const size_t smem = (size_t)((threads / 32 + 2) * E * 4);
  static std::atomic<bool> allowed[64];  // the shared-memory opt-in, per device
  int dev = 0;
  SP24_CUDA_CHECK(cudaGetDevice(&dev));
  if (dev < 0 || dev >= 64 || !allowed[dev].load(std::memory_order_acquire)) {
    SP24_CUDA_CHECK(cudaFuncSetAttribute(order_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 34 * kMostExperts * 4));
    if (dev >= 0 && dev < 64) allowed[dev].store(true, std::memory_order_release);
  }
  return launch_overlapped(order_kernel, dim3((unsigned)blocks), dim3((unsigned)threads), smem, static_cast<cudaStream_t>(stream), (unsigned)blocks, p);
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
  const sp24_status arch = check_arch();
  SP24_RETURN_IF(arch != SP24_OK, arch);
  RowsParams p = {};
  p.T = T; p.K = K; p.rows = rows; p.k = k;
  p.ld_in = ldx * es; p.ld_out = ldo * es;
  p.in = static_cast<const uint8_t*>(x); p.out = static_cast<uint8_t*>(out);
  p.position = position; p.source = source; p.weights = scale; p.sums = out_scale;
  auto run = [&](auto word) {
    using W = decltype(word);
    p.K = K * es / (int64_t)sizeof(W);
    const unsigned threads = row_threads(p.K);
    p.token_blocks = (int)token_blocks(T);
    return launch_overlapped(gather_kernel<W>, dim3(p.token_blocks + clearing_blocks(rows, threads)), dim3(threads), 0, static_cast<cudaStream_t>(stream), 1, p);
  };
  if (whole_vectors(es, K, {x, out}, {ldx, ldo})) return run(uint4{});
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
  const sp24_status arch = check_arch();
  SP24_RETURN_IF(arch != SP24_OK, arch);
  RowsParams p = {};
  p.T = T; p.rows = rows; p.k = k;
  p.ld_y = ldy * es; p.ld_out = ldo * es; p.ld_res = ldr * es;
  p.y = static_cast<const uint8_t*>(y); p.residual = static_cast<const uint8_t*>(residual); p.out = static_cast<uint8_t*>(out);
  p.position = position; p.weights = weights;
  const bool whole = whole_vectors(es, K, {y, out, residual}, {ldy, ldo, residual ? ldr : 0});
  return with_float_type(t, [&](auto type) {
    using Type = typename decltype(type)::type;
    auto run = [&](auto word) {
      using W = decltype(word);
      p.K = K * es / (int64_t)sizeof(W);
      return launch_overlapped(combine_kernel<Type, W>, dim3(token_blocks(T)), dim3(row_threads(p.K)), 0, static_cast<cudaStream_t>(stream), 1, p);
    };
    if (whole) return run(uint4{});
    if constexpr (sizeof(Type) == 4) return run(uint32_t{});
    else return run(uint16_t{});
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
  const sp24_status arch = check_arch();
  SP24_RETURN_IF(arch != SP24_OK, arch);
  RowsParams p = {};
  p.T = T; p.rows = rows; p.k = k;
  p.ld_in = lddo * es; p.ld_y = ldy * es; p.ld_out = lddy * es;
  p.in = static_cast<const uint8_t*>(dout); p.y = static_cast<const uint8_t*>(y); p.out = static_cast<uint8_t*>(dy);
  p.position = position; p.source = source; p.weights = weights; p.sums = dweights;
  const bool whole = whole_vectors(es, K, {dout, y, dy}, {lddo, ldy, lddy});
  return with_float_type(t, [&](auto type) {
    using Type = typename decltype(type)::type;
    auto run = [&](auto word) {
      using W = decltype(word);
      p.K = K * es / (int64_t)sizeof(W);
      const unsigned threads = row_threads(p.K);
      p.token_blocks = (int)token_blocks(T);
      return launch_overlapped(combine_backward_kernel<Type, W>, dim3(p.token_blocks + clearing_blocks(rows, threads)), dim3(threads), 0,
                               static_cast<cudaStream_t>(stream), 1, p);
    };
    if (whole) return run(uint4{});
    if constexpr (sizeof(Type) == 4) return run(uint32_t{});
    else return run(uint16_t{});
  });
}

extern "C" size_t sp24_expert_bias_grad_workspace_bytes(int64_t E, int64_t M, int64_t rows) {
  if (E < 1 || M < 1 || rows < 0) return 0;
  return (size_t)((rows / kBiasRows + E + 1) * M) * 4;
}

extern "C" sp24_status sp24_expert_bias_grad(sp24_dtype t, sp24_act act, int64_t E, int64_t M, int64_t rows, const void* dy, int64_t lddy,
                                             const void* z, int64_t ldz, const int32_t* offsets, float* dbias, void* workspace,
                                             size_t workspace_bytes, void* stream) {
  SP24_RETURN_IF(!is_float_type(t), SP24_ERR_DTYPE);
  SP24_RETURN_IF(!is_act(act), SP24_ERR_UNSUPPORTED);
  SP24_RETURN_IF(E < 1 || E > kMostExperts || M < 1 || M > kMostColumns || rows < 0 || rows > int64_t(1) << 23, SP24_ERR_SHAPE);
  SP24_RETURN_IF(offsets == nullptr || dbias == nullptr || (rows > 0 && (dy == nullptr || (act != SP24_ACT_NONE && z == nullptr))), SP24_ERR_NULL);
  SP24_RETURN_IF(!row_fits(rows, M, lddy) || (act != SP24_ACT_NONE && !row_fits(rows, M, ldz)), SP24_ERR_STRIDE);
  SP24_RETURN_IF(!aligned(dy, elem_bytes(t)) || !aligned(z, elem_bytes(t)) || !aligned(offsets, 4) || !aligned(dbias, 4), SP24_ERR_ALIGN);
  SP24_RETURN_IF(workspace == nullptr || !aligned16(workspace) || workspace_bytes < sp24_expert_bias_grad_workspace_bytes(E, M, rows), SP24_ERR_WORKSPACE);
  const sp24_status arch = check_arch();
  SP24_RETURN_IF(arch != SP24_OK, arch);
  BiasParams p = {rows, M, lddy, ldz, (int)E, dy, z, offsets, static_cast<float*>(workspace), dbias};
  const cudaStream_t s = static_cast<cudaStream_t>(stream);
  const dim3 parts((unsigned)((M + kBiasColumns - 1) / kBiasColumns), (unsigned)(rows / kBiasRows + E + 1));
  const sp24_status st = with_float_type(t, [&](auto type) {
    using Type = typename decltype(type)::type;
    switch (act) {
      case SP24_ACT_RELU: return launch_overlapped(bias_parts_kernel<Type, SP24_ACT_RELU>, parts, dim3(256), 0, s, 1, p);
      case SP24_ACT_GELU: return launch_overlapped(bias_parts_kernel<Type, SP24_ACT_GELU>, parts, dim3(256), 0, s, 1, p);
      case SP24_ACT_SILU: return launch_overlapped(bias_parts_kernel<Type, SP24_ACT_SILU>, parts, dim3(256), 0, s, 1, p);
      case SP24_ACT_GELU_TANH: return launch_overlapped(bias_parts_kernel<Type, SP24_ACT_GELU_TANH>, parts, dim3(256), 0, s, 1, p);
      default: return launch_overlapped(bias_parts_kernel<Type, SP24_ACT_NONE>, parts, dim3(256), 0, s, 1, p);
    }
  });
  SP24_RETURN_IF(st != SP24_OK, st);
  return launch_overlapped(bias_sums_kernel, dim3((unsigned)((M + 255) / 256), (unsigned)E), dim3(256), 0, s, 1, p);
}
