// What the operators on rows share: types, 8-bit codes with a scale for each row, reductions over a row.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "sp24_common.cuh"

namespace sp24 {

constexpr int64_t kMostColumns = int64_t(1) << 30;

inline bool is_float_type(sp24_dtype t) { return t == SP24_F16 || t == SP24_BF16 || t == SP24_F32; }
inline bool is_code_type(sp24_dtype t) { return t == SP24_I8 || is_fp8(t); }
inline bool aligned(const void* p, size_t bytes) { return bytes == 0 || reinterpret_cast<uintptr_t>(p) % bytes == 0; }
// a leading dimension that rows of K elements fit (one row has none)
inline bool row_fits(int64_t rows, int64_t K, int64_t ld) { return rows <= 1 || ld >= K; }

template <typename T>
struct TypeOf {
  using type = T;
};
// f(TypeOf<T>{}) for the type t; with_out_type: T itself or one of the 8-bit types
template <typename F>
inline sp24_status with_float_type(sp24_dtype t, F&& f) {
  switch (t) {
    case SP24_F16: return f(TypeOf<__half>{});
    case SP24_BF16: return f(TypeOf<__nv_bfloat16>{});
    case SP24_F32: return f(TypeOf<float>{});
    default: return SP24_ERR_DTYPE;
  }
}
template <typename T, typename F>
inline sp24_status with_out_type(sp24_dtype t, F&& f) {
  switch (t) {
    case SP24_I8: return f(TypeOf<int8_t>{});
    case SP24_E4M3: return f(TypeOf<__nv_fp8_e4m3>{});
    case SP24_E5M2: return f(TypeOf<__nv_fp8_e5m2>{});
    default: return f(TypeOf<T>{});
  }
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T round_to(float v) {
  if constexpr (sizeof(T) == 4) return v;
  else if constexpr (std::is_same_v<T, __half>) return __float2half_rn(v);
  else return __float2bfloat16_rn(v);
}
template <typename T>
__device__ __forceinline__ float load_weight(const void* w, int f32, int64_t k) {
  return f32 ? static_cast<const float*>(w)[k] : to_float(static_cast<const T*>(w)[k]);
}

// ---- 8-bit results -----------------------------------------------------------------------------------------
template <typename OUT>
constexpr bool is_code = sizeof(OUT) == 1;
template <typename OUT>
constexpr float kLargestCode = std::is_same_v<OUT, int8_t> ? 127.f : std::is_same_v<OUT, __nv_fp8_e4m3> ? 448.f : 57344.f;

// |v| as an integer that grows with it; NaN is above everything, so that a maximum keeps it.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Scale of a row whose values are v * factor with max |v| = top, and what v is multiplied by to give codes.  Rows below 2^-120
// count as zeros (L / top would pass the largest float).  NaN or an infinity anywhere (factor: rstd is NaN or 0 then) gives
// scale NaN; v * NaN is then code 0 as an integer and NaN as a float.
template <typename OUT>
__device__ __forceinline__ float row_scale(float top, float factor, float* inv) {
  constexpr float L = kLargestCode<OUT>;
  if (top < 7.52316385e-37f) {
    *inv = 0.f;
    return 0.f;
  }
  const float scale = top * factor * (1.f / L);
  *inv = scale == scale ? L / top : scale;
  return scale;
}

template <typename OUT>
__device__ __forceinline__ OUT to_code(float v) {
  if constexpr (std::is_same_v<OUT, int8_t>) {
    return (int8_t)max(min(__float2int_rn(v), 127), -127);  // (NaN: 0)
  } else {
    OUT o;
    o.__x = __nv_cvt_float_to_fp8(v, __NV_SATFINITE, std::is_same_v<OUT, __nv_fp8_e4m3> ? __NV_E4M3 : __NV_E5M2);
    return o;
  }
}

// an infinite maximum counts as NaN (where no factor of the row turns it into one)
__device__ __forceinline__ float finite_or_nan(float top) { return top < __int_as_float(0x7f800000) ? top : __int_as_float(0x7fffffff); }

// ---- a row's sum and maximum over a block ----------------------------------------------------------------------
// Two buffers in turn, so that one barrier is enough: whoever writes a buffer again has passed the barrier of the one between,
// which the readers reach behind their reads.
struct RowSums {
  float sum[2][32];
  uint32_t top[2][32];
  // every thread of the block gets the block's sum and maximum
  __device__ __forceinline__ void reduce(float& s, uint32_t& t, int& turn) {
#pragma unroll
    for (int i = 16; i > 0; i >>= 1) s += __shfl_xor_sync(~0u, s, i);
    t = __reduce_max_sync(~0u, t);
    const int warps = blockDim.x >> 5;
    if (warps == 1) return;
    const int lane = threadIdx.x & 31;
    if (lane == 0) {
      sum[turn][threadIdx.x >> 5] = s;
      top[turn][threadIdx.x >> 5] = t;
    }
    __syncthreads();
    s = lane < warps ? sum[turn][lane] : 0.f;
    t = lane < warps ? top[turn][lane] : 0u;
    turn ^= 1;
#pragma unroll
    for (int i = 16; i > 0; i >>= 1) s += __shfl_xor_sync(~0u, s, i);
    t = __reduce_max_sync(~0u, t);
  }
};

// Threads of a block to a row of K elements.
inline int row_threads(int64_t K) {
  int threads = 32;
  while (threads < 1024 && threads * 4 < K) threads *= 2;
  return threads;
}

// out[k] = sum of partial[b * K + k] over b < parts, in an order that parts alone fixes (sp24_rms_norm.cu)
sp24_status column_sums(const float* partial, int64_t parts, int64_t K, float* out, cudaStream_t s);

}  // namespace sp24
