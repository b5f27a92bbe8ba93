// What the operators on rows share: types, 8-bit codes with a scale for each row, reductions over a row.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <type_traits>

#include "sp24_act.cuh"

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

// f(flags as types...) with a member `value` each
template <typename F>
inline auto with_flags(F&& f) { return f(); }
template <typename F, typename... Rest>
inline auto with_flags(F&& f, bool first, Rest... rest) {
  auto go = [&](auto flag) { return with_flags([&](auto... others) { return f(flag, others...); }, rest...); };
  return first ? go(std::true_type{}) : go(std::false_type{});
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

// max(m, |a|, |b|) for m >= 0; NaN stays.
__device__ __forceinline__ float max_abs(float m, float a, float b) {
  asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(a), "f"(b));
  return m;
}

// Scale of a row whose values are v * factor with max |v| = top, and what v is multiplied by to give codes.  Rows below 2^-110
// count as zeros (below 2^-112 L / top could pass the largest float).  NaN or an infinity anywhere (factor: rstd is NaN or 0 then) gives
// scale NaN; v * NaN is then code 0 as an integer and NaN as a float.
template <typename OUT>
__device__ __forceinline__ float row_scale(float top, float factor, float* inv) {
  constexpr float L = kLargestCode<OUT>;
  if (top < 7.7037198e-34f) {
    *inv = 0.f;
    return 0.f;
  }
  const float scale = top * factor * (1.f / L);
  *inv = scale == scale ? L / top : scale;
  return scale;
}

// an infinite maximum counts as NaN (where no factor of the row turns it into one)
__device__ __forceinline__ float finite_or_nan(float top) { return top < __int_as_float(0x7f800000) ? top : __int_as_float(0x7fffffff); }

// ---- a row's sum and maximum over its team -----------------------------------------------------------------------
// A team is blockDim.x threads, a power of two below 32 or whole warps, one of blockDim.y; every thread of it gets the team's sum and
// maximum (of values >= 0).  All threads of a block's warps call it together.  Two buffers in turn, so that one barrier is enough: whoever
// writes a buffer again has passed the barrier of the one between, which the readers reach behind their reads.
constexpr int kMostTeams = 15;  // of several warps: each has a hardware barrier of its own
// The sum is over groups of 32 neighbouring vectors (a warp's v-th ones) and then over the groups, group g first with g + 32 and then by halves, however many
// vectors a thread has, so that a row's bits do not depend on how many other rows there are nor on how they lie.  (Four sums of a warp take six shuffles: each
// of the first two sends away half of what a lane holds.)
struct RowSums {
  float groups[2][64], top[2][32];
  // s: of each of the thread's vectors; the row's sum is in s[0] afterwards
  template <bool SUM, bool TOP, int V>
  __device__ __forceinline__ void reduce(float (&s)[V], float& t, int& turn) {
    if (blockDim.x < 32) {
      if (SUM) {
#pragma unroll
        for (int v = V / 2; v > 0; v /= 2)
#pragma unroll
          for (int i = 0; i < v; ++i) s[i] += s[i + v];
      }
      for (int i = blockDim.x >> 1; i > 0; i >>= 1) {
        if (SUM) s[0] += __shfl_xor_sync(~0u, s[0], i);
        if (TOP) t = max_abs(t, __shfl_xor_sync(~0u, t, i), 0.f);
      }
      return;
    }
    auto sum_over_warp = [&](float& x) {
#pragma unroll
      for (int i = 16; i > 0; i >>= 1) x += __shfl_xor_sync(~0u, x, i);
    };
    auto top_over_warp = [&] { asm volatile("redux.sync.max.abs.NaN.f32 %0, %0, 0xffffffff;" : "+f"(t)); };
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, first = threadIdx.y * warps;
    constexpr int G = V;  // groups of a warp: at most 64 of all teams (32 warps with one or two, 16 with four)
    if constexpr (SUM && V == 4) {  // (teams of many warps); of lanes 8 v on: the v-th group's sum
      const bool hi = lane & 16, odd = lane & 8;
      const float a = (hi ? s[2] : s[0]) + __shfl_xor_sync(~0u, hi ? s[0] : s[2], 16), b = (hi ? s[3] : s[1]) + __shfl_xor_sync(~0u, hi ? s[1] : s[3], 16);
      s[0] = (odd ? b : a) + __shfl_xor_sync(~0u, odd ? a : b, 8);
#pragma unroll
      for (int i = 4; i > 0; i >>= 1) s[0] += __shfl_xor_sync(~0u, s[0], i);
      if ((lane & 7) == 0) groups[turn][G * first + (lane >> 3) * warps + warp] = s[0];
    } else if constexpr (SUM) {
#pragma unroll
      for (int v = 0; v < V; ++v) sum_over_warp(s[v]);
    }
    if (TOP) top_over_warp();
    if (V != 4 && warps == 1) {
      if (SUM && V == 2) s[0] += s[V - 1];
      return;
    }
    if (lane == 0) {
      if (SUM && V != 4) {
#pragma unroll
        for (int v = 0; v < V; ++v) groups[turn][G * first + v * warps + warp] = s[v];
      }
      if (TOP) top[turn][first + warp] = t;
    }
    asm volatile("bar.sync %0, %1;" ::"r"(threadIdx.y + 1), "r"(blockDim.x) : "memory");
    if (SUM) {
      s[0] = lane < G * warps ? groups[turn][G * first + lane] : 0.f;
      if (G * warps > 32) s[0] += lane + 32 < G * warps ? groups[turn][G * first + lane + 32] : 0.f;
    }
    if (TOP) t = lane < warps ? top[turn][first + lane] : 0.f;
    turn ^= 1;
    if (SUM) sum_over_warp(s[0]);
    if (TOP) top_over_warp();
  }
};

// ---- rows in registers --------------------------------------------------------------------------------------------
// A thread has V vectors of a row, number threadIdx.x + v * blockDim.x: 16 bytes of the type T that the operator works on, N elements, N / 2
// pairs.
template <typename T>
constexpr int kVector = 16 / sizeof(T);
template <typename T>
using Pairs = float2[kVector<T> / 2];

template <typename T>
__device__ __forceinline__ void unpack(const uint4& w, Pairs<T>& f) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  if constexpr (sizeof(T) == 4) {
    f[0] = make_float2(__uint_as_float(w.x), __uint_as_float(w.y));
    f[1] = make_float2(__uint_as_float(w.z), __uint_as_float(w.w));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same_v<T, __half>) f[i] = __half22float2(*reinterpret_cast<const __half2*>(&x[i]));
      else f[i] = make_float2(__uint_as_float(x[i] << 16), __uint_as_float(x[i] & 0xffff0000u));
    }
  }
}
template <typename T>
__device__ __forceinline__ uint4 pack(const Pairs<T>& f) {
  if constexpr (sizeof(T) == 4) {
    return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
  } else {
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (std::is_same_v<T, __half>) {
        const __half2 v = __float22half2_rn(f[i]);
        x[i] = *reinterpret_cast<const uint32_t*>(&v);
      } else {
        const __nv_bfloat162 v = __float22bfloat162_rn(f[i]);
        x[i] = *reinterpret_cast<const uint32_t*>(&v);
      }
    }
    return make_uint4(x[0], x[1], x[2], x[3]);
  }
}
// a + b element by element, rounded to T
template <typename T>
__device__ __forceinline__ uint4 add_packed(const uint4& a, const uint4& b) {
  const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
  uint32_t z[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) {
      z[i] = __float_as_uint(__uint_as_float(x[i]) + __uint_as_float(y[i]));
    } else if constexpr (std::is_same_v<T, __half>) {
      const __half2 v = __hadd2(*reinterpret_cast<const __half2*>(&x[i]), *reinterpret_cast<const __half2*>(&y[i]));
      z[i] = *reinterpret_cast<const uint32_t*>(&v);
    } else {
      const __nv_bfloat162 v = __hadd2(*reinterpret_cast<const __nv_bfloat162*>(&x[i]), *reinterpret_cast<const __nv_bfloat162*>(&y[i]));
      z[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
  }
  return make_uint4(z[0], z[1], z[2], z[3]);
}

// ---- rows that start between 16-byte boundaries ----------------------------------------------------------------------------------
// Bytes `o` (below 4 * WORDS; a multiple of BYTES) and on of the 8 * WORDS bytes {lo, hi}.
template <int BYTES, int WORDS>
__device__ __forceinline__ void from_byte(const uint32_t (&lo)[WORDS], const uint32_t (&hi)[WORDS], int o, uint32_t (&out)[WORDS]) {
  uint32_t w[2 * WORDS];
#pragma unroll
  for (int i = 0; i < WORDS; ++i) {
    w[i] = lo[i];
    w[WORDS + i] = hi[i];
  }
#pragma unroll
  for (int by = WORDS / 2; by > 0; by /= 2) {
    const bool shift = o & (4 * by);
#pragma unroll
    for (int i = 0; i + by < 2 * WORDS; ++i) w[i] = shift ? w[i + by] : w[i];
  }
#pragma unroll
  for (int i = 0; i < WORDS; ++i) out[i] = BYTES % 4 == 0 ? w[i] : __funnelshift_r(w[i], w[i + 1], 8 * (o & 3));
}

// Where the vectors of a row lie: number i holds the elements from i * N - shift on, so that the words of a row whose first element lies
// `shift` elements behind a boundary are whole vectors (WHOLE: all rows start at boundaries and end with a vector, shift is 0).
template <typename E, int N>
__device__ __forceinline__ int shift_of(const E* row) {
  return (int)(reinterpret_cast<uintptr_t>(row) / sizeof(E) % N);
}

// The words that vector i of a row of K elements lies in: one if the vectors lie at boundaries, else two, of which the vector is made where it is used, so that
// nothing waits for them before.  A word is read if one of the row's elements is in it: the bytes beside them are in the same 16, and not used.
template <bool WHOLE>
struct Words {
  uint4 lo, hi;
};
template <>
struct Words<true> {
  uint4 lo;
};
template <typename T>
__device__ __forceinline__ int behind_words(const T* row, int shift) {  // bytes that the vectors lie behind the words
  return (int)(reinterpret_cast<uintptr_t>(row - shift) & 15);
}
template <bool WHOLE, typename T>
__device__ __forceinline__ void load_words(Words<WHOLE>& to, const T* row, int i, int K, int shift) {
  constexpr int N = kVector<T>;
  if constexpr (WHOLE) {
    to.lo = i * N < K ? __ldcs(reinterpret_cast<const uint4*>(row) + i) : make_uint4(0, 0, 0, 0);
  } else {
    const int o = behind_words(row, shift);
    const uint4* words = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(row - shift) - o);
    auto word = [&](int j) {
      const int e = j * N - shift - o / (int)sizeof(T);  // the word's first element
      return e < K && e + N > 0 ? words[j] : make_uint4(0, 0, 0, 0);
    };
    to.lo = word(i);
    if (o) to.hi = word(i + 1);
  }
}
// The vector, zeros where the row has no elements.
template <bool WHOLE, typename T>
__device__ __forceinline__ uint4 vector_of(const Words<WHOLE>& from, const T* row, int i, int K, int shift) {
  if constexpr (WHOLE) {
    return from.lo;
  } else {
    constexpr int N = kVector<T>;
    const int first = i * N - shift, o = behind_words(row, shift);
    uint32_t w[4] = {from.lo.x, from.lo.y, from.lo.z, from.lo.w};
    if (o) {
      const uint32_t lo[4] = {w[0], w[1], w[2], w[3]}, hi[4] = {from.hi.x, from.hi.y, from.hi.z, from.hi.w};
      from_byte<(int)sizeof(T)>(lo, hi, o, w);
    }
    if (first < 0 || first + N > K) {
      T* e = reinterpret_cast<T*>(w);
      const T zero = {};
#pragma unroll
      for (int n = 0; n < N; ++n)
        if ((unsigned)(first + n) >= (unsigned)K) e[n] = zero;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
}
// Both at once, where registers count: the operators that hold rows (words apart: spills; norm bf16 8192 x 12287 -> e4m3 252, 296 us, silu f16
// 4099 x 5461 43, 51).  gated_act_backward, which holds none, has its loads apart: f16 4099 x 5461 75, 67 us.
template <bool WHOLE, typename T>
__device__ __forceinline__ uint4 load_vector(const T* row, int i, int K, int shift) {
  constexpr int N = kVector<T>;
  if (WHOLE) return i * N < K ? __ldcs(reinterpret_cast<const uint4*>(row) + i) : make_uint4(0, 0, 0, 0);
  const int first = i * N - shift;  // its first element's number
  const int o = behind_words(row, shift), behind = o / (int)sizeof(T);
  const uint4* words = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(row - shift) - o);
  auto word = [&](int j) {
    const int e = j * N - shift - behind;  // the word's first element
    return e < K && e + N > 0 ? words[j] : make_uint4(0, 0, 0, 0);
  };
  uint4 a = word(i);
  uint32_t w[4] = {a.x, a.y, a.z, a.w};
  if (o) {
    a = word(i + 1);
    const uint32_t lo[4] = {w[0], w[1], w[2], w[3]}, hi[4] = {a.x, a.y, a.z, a.w};
    from_byte<(int)sizeof(T)>(lo, hi, o, w);
  }
  if (first < 0 || first + N > K) {
    T* e = reinterpret_cast<T*>(w);
    const T zero = {};
#pragma unroll
    for (int n = 0; n < N; ++n)
      if ((unsigned)(first + n) >= (unsigned)K) e[n] = zero;
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// Vector i of a row of K elements, 4 * WORDS bytes of E, to the row: as one word if it lies at a boundary, else by elements.
template <bool WHOLE, typename E, int WORDS>
__device__ __forceinline__ void store_words(E* row, int i, int K, int shift, const uint32_t (&w)[WORDS]) {
  constexpr int N = 4 * WORDS / sizeof(E);
  const int first = i * N - (WHOLE ? 0 : shift);
  if (WHOLE ? first < K : first >= 0 && first + N <= K && reinterpret_cast<uintptr_t>(row - shift) % (4 * WORDS) == 0) {
    if constexpr (WORDS == 4) *reinterpret_cast<uint4*>(row + first) = make_uint4(w[0], w[1], w[2], w[3]);
    else if constexpr (WORDS == 2) *reinterpret_cast<uint2*>(row + first) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(row + first) = w[0];
    return;
  }
  if (WHOLE) return;
  const E* e = reinterpret_cast<const E*>(w);
#pragma unroll
  for (int n = 0; n < N; ++n)
    if ((unsigned)(first + n) < (unsigned)K) row[first + n] = e[n];
}
template <bool WHOLE, typename T>
__device__ __forceinline__ void store_vector(T* row, int i, int K, int shift, const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  store_words<WHOLE>(row, i, K, shift, w);
}
// ... as N codes
template <bool WHOLE, typename OUT, int PAIRS>
__device__ __forceinline__ void store_codes(OUT* row, int i, int K, int shift, const float2 (&f)[PAIRS]) {
  constexpr int N = 2 * PAIRS;
  uint32_t w[N / 4];
#pragma unroll
  for (int n = 0; n < N / 4; ++n) {
    const float2 lo = f[2 * n], hi = f[2 * n + 1];
    if constexpr (std::is_same_v<OUT, int8_t>) {  // (NaN: 0.  |v| is at most 127 (1 + 2^-22), which rounds to no more than 127.)
      asm("cvt.pack.sat.s8.s32.b32 %0, %1, %2, 0;" : "=r"(w[n]) : "r"(__float2int_rn(hi.y)), "r"(__float2int_rn(hi.x)));
      asm("cvt.pack.sat.s8.s32.b32 %0, %1, %2, %0;" : "+r"(w[n]) : "r"(__float2int_rn(lo.y)), "r"(__float2int_rn(lo.x)));
    } else {
      constexpr __nv_fp8_interpretation_t kind = std::is_same_v<OUT, __nv_fp8_e4m3> ? __NV_E4M3 : __NV_E5M2;
      w[n] = __nv_cvt_float2_to_fp8x2(lo, __NV_SATFINITE, kind) | (uint32_t)__nv_cvt_float2_to_fp8x2(hi, __NV_SATFINITE, kind) << 16;
    }
  }
  store_words<WHOLE>(row, i, K, shift, w);
}

// Vectors that hold a row of K elements wherever it starts.
inline int64_t row_vectors(int64_t K, size_t es, bool whole) { return ((K + (whole ? 0 : 16 / (int64_t)es - 1)) * (int64_t)es + 15) / 16; }

// Whether the rows start at `bytes` boundaries (an absent matrix does).
inline bool whole_rows(const void* base, int64_t rows, int64_t ld, size_t es, size_t bytes) {
  return !base || (aligned(base, bytes) && (rows <= 1 || (size_t)ld * es % bytes == 0));
}

// Teams, blocks and vectors to a thread for rows that a team holds in registers: a block to an SM, as many teams to a block as its threads
// and the SM's rows allow.  Each thread has two vectors on their way where there are rows enough, one where an SM has few; four in the
// longest rows.  (Registers: 1024 threads with one vector, 768 with two, 512 with four.)
constexpr int team_threads(int v) { return v == 1 ? 1024 : v == 2 ? 768 : 512; }
constexpr int64_t kMostTeamVectors = 4 * team_threads(4);
struct TeamLaunch {
  dim3 grid, block;
  int v;
  // with_two: threads of a block with two vectors each, where they suffice; from_rows: rows of an SM from which on they have two
  TeamLaunch(int64_t rows, int64_t vectors, int from_rows, int with_two = team_threads(2)) {
    const int64_t sms = sm_count();
    v = vectors > 2 * team_threads(2) ? 4 : vectors > team_threads(1) || rows > from_rows * sms ? 2 : 1;
    const int64_t most = v == 2 && vectors <= 2 * with_two ? with_two : team_threads(v);
    const int64_t lanes = (vectors + v - 1) / v;
    int64_t team = (lanes + 31) / 32 * 32;
    if (lanes < 32)
      for (team = 4; team < lanes; team *= 2) {
      }
    int64_t teams = most / team;
    if (team > 32 && teams > kMostTeams) teams = kMostTeams;
    const int64_t each = (rows + sms - 1) / sms, whole_warp = team < 32 ? 32 / team : 1;  // rows of an SM; teams of a warp
    if (teams > each) teams = (each + whole_warp - 1) / whole_warp * whole_warp;
    block = dim3((unsigned)team, (unsigned)teams);
    int64_t blocks = (rows + teams - 1) / teams;
    if (blocks > sms) blocks = sms;
    grid = dim3((unsigned)blocks);
  }
};

// out[k] = sum of partial[b * K + k] over b < parts, in an order that parts alone fixes (sp24_rms_norm.cu)
sp24_status column_sums(const float* partial, int64_t parts, int64_t K, float* out, cudaStream_t s);

}  // namespace sp24
