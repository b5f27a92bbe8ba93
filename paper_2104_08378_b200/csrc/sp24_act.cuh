// The activations and their slopes, in FP32, as the streaming kernels and the epilogue of the products use them.
#pragma once

#include "sp24_common.cuh"

namespace sp24 {

inline bool is_act(int act) { return act >= SP24_ACT_NONE && act <= SP24_ACT_GELU_TANH; }

// ---- pairs: two FP32 operations of one instruction, each rounded by itself --------------------------------------------------
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  asm("{ .reg .b64 x, y; mov.b64 x, {%0, %1}; mov.b64 y, {%2, %3}; mul.rn.f32x2 x, x, y; mov.b64 {%0, %1}, x; }" : "+f"(a.x), "+f"(a.y) : "f"(b.x), "f"(b.y));
  return a;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  asm("{ .reg .b64 x, y, z; mov.b64 x, {%2, %3}; mov.b64 y, {%4, %5}; mov.b64 z, {%0, %1}; fma.rn.f32x2 z, x, y, z; mov.b64 {%0, %1}, z; }"
      : "+f"(c.x), "+f"(c.y)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return c;
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// ---- activations, two values at a time ----------------------------------------------------------------------------------------------
// 2^v and 1 / v of the special-function units, without the instructions that keep results below 2^-126 (which become 0: next to the 1 they are added to, or as a
// factor of a value below 2^7, they do not count).  They set the pace: two of them to an activation, of which a multiprocessor does sixteen a
// cycle.
__device__ __forceinline__ float exp2_fast(float v) {
  asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(v));
  return v;
}
__device__ __forceinline__ float reciprocal_fast(float v) {
  asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(v));
  return v;
}
constexpr float kLog2e = 1.4426950408889634f;

// Phi of the normal distribution: Phi(-|z|) = exp(-z^2 / 2) t (q1 + q2 t + ... + q8 t^7) with t = 1 / (1 + 0.304 |z|), which a positive z subtracts from 1.
// The polynomial is a fit of exp(z^2 / 2) Phi(-|z|) by Remez's exchange with the smallest relative error, 8.4e-8, for |z| <= 13.5 (beyond,
// exp(-z^2 / 2) is 0).  So the tail keeps its leading bits, which a fit with an absolute error does not: at most 2^-19 + 1.25 z^2 2^-24 of the value are lost
// (t and its powers, the exponential, and z^2 / 2 log2(e) rounded three times).  `density`: exp(-z^2 / 2), which the slope needs as well.
__device__ __forceinline__ float2 normal_cdf(float2 z, float2* density) {
  constexpr float p = 0.304f;
  const float2 t = make_float2(reciprocal_fast(fmaf(fabsf(z.x), p, 1.f)), reciprocal_fast(fmaf(fabsf(z.y), p, 1.f)));
  const float2 square = mul2(mul2(z, both(-0.5f * kLog2e)), z);
  *density = make_float2(exp2_fast(square.x), exp2_fast(square.y));
  float2 poly = fma2(t, both(3.6857929563e-02f), both(-1.5529669541e-01f));
  poly = fma2(t, poly, both(1.9218532803e-01f));
  poly = fma2(t, poly, both(-4.3127016641e-02f));
  poly = fma2(t, poly, both(1.2355224943e-01f));
  poly = fma2(t, poly, both(1.0242285091e-01f));
  poly = fma2(t, poly, both(1.2217071321e-01f));
  poly = fma2(t, poly, both(1.2123468153e-01f));
  const float2 tail = mul2(mul2(t, poly), *density);  // Phi(-|z|)
  return make_float2(z.x < 0.f ? tail.x : 1.f - tail.x, z.y < 0.f ? tail.y : 1.f - tail.y);
}

// 1 / (1 + exp(-v)) of v = z * factor / log2(e).  (exp(-v) = inf gives 0.)
__device__ __forceinline__ float2 logistic_of(float2 v_log2e) {
  const float2 e = make_float2(exp2_fast(-v_log2e.x), exp2_fast(-v_log2e.y));
  return make_float2(reciprocal_fast(1.f + e.x), reciprocal_fast(1.f + e.y));
}

// gelu with tanh: (1 + tanh(u)) / 2 = 1 / (1 + exp(-2 u)), u = sqrt(2 / pi) (z + 0.044715 z^3).  (z^2 is limited where the logistic has
// long been 0 or 1, so that 0 times it is 0.)
__device__ __forceinline__ float2 limited_square(float2 z) {
  const float2 s = mul2(z, z);
  return make_float2(fminf(s.x, 1e9f), fminf(s.y, 1e9f));
}
__device__ __forceinline__ float2 tanh_logistic(float2 z) {
  constexpr float c = 1.5957691216f * kLog2e;  // 2 sqrt(2 / pi), for 2^v
  return logistic_of(mul2(z, fma2(both(c * 0.044715f), limited_square(z), both(c))));
}

template <int ACT>
__device__ __forceinline__ float2 act_value(float2 z) {
  if (ACT == SP24_ACT_RELU) return make_float2(z.x < 0.f ? 0.f : z.x, z.y < 0.f ? 0.f : z.y);  // (NaN stays)
  if (ACT == SP24_ACT_GELU) {
    float2 density;
    return mul2(z, normal_cdf(z, &density));
  }
  if (ACT == SP24_ACT_SILU) return mul2(z, logistic_of(mul2(z, both(kLog2e))));
  if (ACT == SP24_ACT_GELU_TANH) return mul2(z, tanh_logistic(z));
  return z;
}

// act(z), and act'(z) in *slope
template <int ACT>
__device__ __forceinline__ float2 act_and_slope(float2 z, float2* slope) {
  if (ACT == SP24_ACT_RELU) {
    slope->x = z.x > 0.f ? 1.f : (z.x <= 0.f ? 0.f : z.x);
    slope->y = z.y > 0.f ? 1.f : (z.y <= 0.f ? 0.f : z.y);
    return act_value<ACT>(z);
  }
  if (ACT == SP24_ACT_GELU) {
    float2 density;
    const float2 cdf = normal_cdf(z, &density);
    *slope = fma2(mul2(z, density), both(0.39894228f), cdf);
    return mul2(z, cdf);
  }
  if (ACT == SP24_ACT_SILU || ACT == SP24_ACT_GELU_TANH) {  // z p(v): p + p (1 - p) z v'
    const float2 p = ACT == SP24_ACT_SILU ? logistic_of(mul2(z, both(kLog2e))) : tanh_logistic(z);
    const float2 q = mul2(mul2(p, make_float2(1.f - p.x, 1.f - p.y)), z);
    *slope = ACT == SP24_ACT_SILU ? make_float2(q.x + p.x, q.y + p.y)
                                  : fma2(q, fma2(both(1.5957691216f * 0.134145f), limited_square(z), both(1.5957691216f)), p);
    return mul2(z, p);
  }
  *slope = both(1.f);
  return z;
}

// f(Act<ACT>{}) for the activation `act`
template <int ACT>
struct Act {
  static constexpr int value = ACT;
};
template <typename F>
inline auto with_act(int act, F&& f) {
  switch (act) {
    case SP24_ACT_RELU: return f(Act<SP24_ACT_RELU>{});
    case SP24_ACT_GELU: return f(Act<SP24_ACT_GELU>{});
    case SP24_ACT_SILU: return f(Act<SP24_ACT_SILU>{});
    case SP24_ACT_GELU_TANH: return f(Act<SP24_ACT_GELU_TANH>{});
    default: return f(Act<SP24_ACT_NONE>{});
  }
}

// the same on the device, for an activation that all threads share
template <typename F>
__device__ __forceinline__ void device_with_act(int act, F&& f) {
  if (act == SP24_ACT_SILU) f(Act<SP24_ACT_SILU>{});
  else if (act == SP24_ACT_GELU) f(Act<SP24_ACT_GELU>{});
  else if (act == SP24_ACT_GELU_TANH) f(Act<SP24_ACT_GELU_TANH>{});
  else if (act == SP24_ACT_RELU) f(Act<SP24_ACT_RELU>{});
  else f(Act<SP24_ACT_NONE>{});
}

}  // namespace sp24
