// The activations and their slopes, in FP32, as the streaming kernels and the epilogue of the products use them.
#pragma once

#include "sp24_common.cuh"

namespace sp24 {

inline bool is_act(int act) { return act >= SP24_ACT_NONE && act <= SP24_ACT_GELU_TANH; }

// Phi(z) = (1 + erf(z / sqrt 2)) / 2 by Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26 (absolute error of
// erf at most 1.5e-7; half of that here): erfc(x) = (a1 t + ... + a5 t^5) exp(-x^2), t = 1 / (1 + p x), for x >= 0.  `density`:
// exp(-z^2 / 2) / sqrt(2 pi), which the slope needs as well.  One exponential and one reciprocal.
__device__ __forceinline__ float normal_cdf(float z, float* density) {
  const float t = __fdividef(1.f, fmaf(fabsf(z), 0.3275911f * 0.70710678f, 1.f));
  const float e = __expf(-0.5f * z * z);
  float poly = fmaf(t, 1.061405429f, -1.453152027f);
  poly = fmaf(t, poly, 1.421413741f);
  poly = fmaf(t, poly, -0.284496736f);
  poly = fmaf(t, poly, 0.254829592f);
  const float tail = 0.5f * t * poly * e;  // Phi(-|z|)
  *density = 0.39894228f * e;
  return z < 0.f ? tail : 1.f - tail;
}

// 1 / (1 + exp(-v)).  (exp(-v) = inf gives 0; __fdividef gives 0 for divisors above 2^126 as well.)
__device__ __forceinline__ float logistic(float v) { return __fdividef(1.f, 1.f + __expf(-v)); }

// gelu with tanh: (1 + tanh(u)) / 2 = logistic(2 u), u = sqrt(2 / pi) (z + 0.044715 z^3).  (z^2 is limited where the logistic has
// long been 0 or 1, so that 0 times it is 0.)
__device__ __forceinline__ float limited_square(float z) { return fminf(z * z, 1e9f); }
__device__ __forceinline__ float tanh_argument(float z) { return z * fmaf(1.5957691f * 0.044715f, limited_square(z), 1.5957691f); }

template <int ACT>
__device__ __forceinline__ float act_value(float z) {
  if (ACT == SP24_ACT_RELU) return z < 0.f ? 0.f : z;  // (NaN stays)
  if (ACT == SP24_ACT_GELU) {
    float density;
    return z * normal_cdf(z, &density);
  }
  if (ACT == SP24_ACT_SILU) return z * logistic(z);
  if (ACT == SP24_ACT_GELU_TANH) return z * logistic(tanh_argument(z));
  return z;
}

// act(z), and act'(z) in *slope
template <int ACT>
__device__ __forceinline__ float act_and_slope(float z, float* slope) {
  if (ACT == SP24_ACT_RELU) {
    *slope = z > 0.f ? 1.f : (z <= 0.f ? 0.f : z);
    return z < 0.f ? 0.f : z;
  }
  if (ACT == SP24_ACT_GELU) {
    float density;
    const float cdf = normal_cdf(z, &density);
    *slope = fmaf(z, density, cdf);
    return z * cdf;
  }
  if (ACT == SP24_ACT_SILU) {
    const float p = logistic(z);
    *slope = p * fmaf(z, 1.f - p, 1.f);
    return z * p;
  }
  if (ACT == SP24_ACT_GELU_TANH) {
    const float p = logistic(tanh_argument(z));
    *slope = fmaf(p * (1.f - p) * z, fmaf(1.5957691f * 0.134145f, limited_square(z), 1.5957691f), p);
    return z * p;
  }
  *slope = 1.f;
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
