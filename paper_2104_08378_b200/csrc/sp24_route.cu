// Routing of tokens to experts, and its gradient.
#include <cfloat>

#include "sp24_rows.cuh"

namespace sp24 {
namespace {

constexpr int kMostExperts = 1024, kMostChosen = 32, kMostGroups = 32;
constexpr int kRouteWarps = 8;

struct RouteParams {
  int64_t T, ld;
  int E, k, groups, group_experts, top_groups;
  int sigmoid, top2, renorm;
  float scale;
  const void* logits;
  const float* bias;
  float* weights;
  int32_t* experts;
};

// Floats as unsigned integers of the same order; 0 is below all of them.
__device__ __forceinline__ uint32_t order_key(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);  // (-0 counts as 0)
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7fffffffu : ~k); }
constexpr uint32_t kDeadKey = 0x007fffffu;  // of -infinity, and what NaN is set to: never chosen

template <typename T>
__device__ __forceinline__ float logit(const void* row, int64_t e) { return to_float(static_cast<const T*>(row)[e]); }

// One warp has a token; lane i has experts i, i + 32, ... (V of them, fewer than 32 V experts).
// The choice is k rounds of the largest key, the lowest index first.  Where FP32 does not tell two values apart, FP64 does.
template <int V>
struct Choice {
  uint32_t key[V];
  // the largest key of the warp and its lowest expert; false if all are dead
  __device__ __forceinline__ bool best(int lane, uint32_t& top, int& expert) const {
    uint32_t m = key[0];
#pragma unroll
    for (int v = 1; v < V; ++v) m = max(m, key[v]);
    top = __reduce_max_sync(~0u, m);
    if (top <= kDeadKey) return false;
    int e = INT_MAX;
#pragma unroll
    for (int v = V - 1; v >= 0; --v)
      if (key[v] == top) e = v * 32 + lane;
    expert = __reduce_min_sync(~0u, e);
    return true;
  }
  __device__ __forceinline__ void take(int lane, int expert) {
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (v * 32 + lane == expert) key[v] = 0;
  }
};

__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
  for (int i = 16; i > 0; i >>= 1) v += __shfl_xor_sync(~0u, v, i);
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int i = 16; i > 0; i >>= 1) v += __shfl_xor_sync(~0u, v, i);
  return v;
}
__device__ __forceinline__ double warp_max(double v) {
#pragma unroll
  for (int i = 16; i > 0; i >>= 1) v = fmax(v, __shfl_xor_sync(~0u, v, i));
  return v;
}

// The whole choice in FP64, for the tokens of which FP32 cannot tell it: rare, so kept out of the way.
template <typename T, int V>
__device__ __noinline__ void choose64(const RouteParams& p, const void* row, float top_logit, int lane, int32_t* chosen) {
  double c[V], by[V];
  double sum = 0.0;
  for (int v = 0; v < V; ++v) {
    const int e = v * 32 + lane;
    const float l = e < p.E ? logit<T>(row, e) : -INFINITY;
    by[v] = p.sigmoid ? 1.0 / (1.0 + exp(-(double)l)) : exp((double)l - (double)top_logit);
    c[v] = l > -INFINITY ? (double)l : -INFINITY;  // (NaN too)
    if (l > -INFINITY) sum += by[v];
  }
  sum = p.sigmoid ? 1.0 : warp_sum(sum);
  for (int v = 0; v < V; ++v) {
    const int e = v * 32 + lane;
    const double b = p.bias && e < p.E ? (double)p.bias[e] : 0.0;
    by[v] = c[v] > -INFINITY && by[v] / sum + b > -INFINITY ? by[v] / sum + b : -INFINITY;
    if (p.bias) c[v] = by[v];
  }
  if (p.groups > 1) {
    double mine = -INFINITY;  // of group `lane`
    for (int g = 0; g < p.groups; ++g) {
      double one = -INFINITY, two = -INFINITY;
      for (int v = 0; v < V; ++v) {
        const int e = v * 32 + lane;
        const double x = p.top2 ? by[v] : c[v];
        if (e / p.group_experts == g && e < p.E) {
          two = fmax(two, fmin(one, x));
          one = fmax(one, x);
        }
      }
#pragma unroll
      for (int i = 16; i > 0; i >>= 1) {
        const double a = __shfl_xor_sync(~0u, one, i), b = __shfl_xor_sync(~0u, two, i);
        two = fmax(fmin(one, a), fmax(two, b));
        one = fmax(one, a);
      }
      if (g == lane) mine = p.top2 && two > -INFINITY ? one + two : one;
    }
    bool open = lane < p.groups, kept = false;
    for (int i = 0; i < p.top_groups; ++i) {
      const double top = warp_max(open ? mine : -INFINITY);
      const uint32_t at = __ballot_sync(~0u, open && mine == top);
      if (at && lane == __ffs(at) - 1) { open = false; kept = true; }
    }
    const uint32_t groups = __ballot_sync(~0u, kept);
    for (int v = 0; v < V; ++v)
      if (!(groups >> ((v * 32 + lane) / p.group_experts & 31) & 1)) c[v] = -INFINITY;
  }
  for (int i = 0; i < p.k; ++i) {
    double m = c[0];
    for (int v = 1; v < V; ++v) m = fmax(m, c[v]);
    m = warp_max(m);
    int e = INT_MAX;
    for (int v = V - 1; v >= 0; --v)
      if (c[v] == m) e = v * 32 + lane;
    e = __reduce_min_sync(~0u, e);
    if (!(m > -INFINITY)) e = -1;
    if (lane == 0) chosen[i] = e;
    for (int v = 0; v < V; ++v)
      if (v * 32 + lane == e) c[v] = -INFINITY;
  }
  __syncwarp();
}

// Lane i's candidate among the m best by FP32 (m <= 32; none of the others can be among them): its place by s + b in FP64, the lower index first.
template <typename T, int V>
__device__ __noinline__ int order64(const RouteParams& p, const void* row, float top_logit, int lane, int m, int expert) {
  double sum = 1.0, c = -INFINITY;
  if (!p.sigmoid) {
    sum = 0.0;
    for (int v = 0; v < V; ++v) {
      const int e = v * 32 + lane;
      const float l = e < p.E ? logit<T>(row, e) : -INFINITY;
      if (l > -INFINITY) sum += exp((double)l - (double)top_logit);
    }
    sum = warp_sum(sum);
  }
  if (lane < m) {
    const double l = (double)logit<T>(row, expert);
    c = (p.sigmoid ? 1.0 / (1.0 + exp(-l)) : exp(l - (double)top_logit) / sum) + (double)p.bias[expert];
  }
  int place = 0;
  for (int i = 0; i < m; ++i) {
    const double other = __shfl_sync(~0u, c, i);
    const int e = __shfl_sync(~0u, expert, i);
    place += other > c || (other == c && e < expert);
  }
  // the i-th place's expert to lane i
  int mine = -1;
  for (int i = 0; i < m; ++i) {
    const uint32_t at = __ballot_sync(~0u, lane < m && place == i);
    const int e = __shfl_sync(~0u, expert, __ffs(at) - 1);
    if (lane == i) mine = e;
  }
  return mine;
}

// What bounds it: instructions, about 500 a token of 256 experts with groups and a bias (the scores a tenth of it, eight rounds of choosing half), so nothing is done
// per expert that can be done once: the bias and the groups of a lane's experts stay in registers over its tokens, scores for the choice come from the
// special-function units (the weights are computed again, exactly, for the chosen), the best of a group is found in shared memory by 32 / groups lanes
// each.  BIAS, GROUPS: kernels without either carry none of it.
template <typename T, int V, bool BIAS, bool GROUPS>
__global__ void __launch_bounds__(32 * kRouteWarps) route_kernel(const RouteParams p) {
  __shared__ int32_t chosen_of[kRouteWarps][kMostChosen];
  extern __shared__ float values_of[];  // GROUPS: E for each warp
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int32_t* chosen = chosen_of[warp];
  float* values = values_of + warp * p.E;
  wait_for_stream();
  const bool two = GROUPS && p.top2, scores = BIAS || two, total = !p.sigmoid && !p.renorm;
  float bias[V], bias_size = 0.f;
  uint32_t group_bit[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int e = v * 32 + lane;
    if (BIAS) {
      bias[v] = e < p.E ? p.bias[e] : -INFINITY;
      bias_size = fmaxf(bias_size, fabsf(bias[v]) < INFINITY ? fabsf(bias[v]) : 0.f);
    }
    if (GROUPS) group_bit[v] = 1u << ((e < p.E ? e / p.group_experts : 0) & 31);
  }
  if (BIAS) asm volatile("redux.sync.max.f32 %0, %0, 0xffffffff;" : "+f"(bias_size));
  // lanes to a group: a power of two
  int parts = 1;
  if (GROUPS)
    while (2 * parts * p.groups <= 32) parts *= 2;
  for (int64_t t = (int64_t)blockIdx.x * kRouteWarps + warp; t < p.T; t += (int64_t)gridDim.x * kRouteWarps) {
    const void* row = static_cast<const T*>(p.logits) + t * p.ld;
    float l[V];
    float top = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int e = v * 32 + lane;
      l[v] = e < p.E ? logit<T>(row, e) : -INFINITY;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
      nan |= l[v] != l[v];
      top = fmaxf(top, l[v]);
    }
    asm volatile("redux.sync.max.f32 %0, %0, 0xffffffff;" : "+f"(top));
    nan = __any_sync(~0u, nan) || (!p.sigmoid && top == INFINITY);
    Choice<V> choice;
    float inv = 1.f, error = 0.f;  // of two scores' difference
    bool sure = true;
    if (total) {
      float sum = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) sum += l[v] > -INFINITY ? expf(l[v] - top) : 0.f;
      inv = 1.f / warp_sum(sum);
    }
    if (scores) {
      // For the choice: off by less than 1.5 2^-22 (sigmoid: half a step of the sum, a step of the reciprocal, a quarter of the exponential's two) or
      // 2^-20 of the largest (softmax: the exponential's argument, up to d below the largest's, rounded twice, (d + 8) exp(-d) 2^-23 at most, and the sum).
      float c[V];
      if (p.sigmoid) {
        error = 2.f * 1.5f * 0x1p-22f;
#pragma unroll
        for (int v = 0; v < V; ++v) c[v] = reciprocal_fast(1.f + exp2_fast(-kLog2e * l[v]));
      } else {
        float sum = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          c[v] = l[v] > -INFINITY ? exp2_fast(kLog2e * (l[v] - top)) : 0.f;
          sum += c[v];
        }
        const float part = 1.f / warp_sum(sum);
        error = 2.f * 0x1p-20f * part;  // (the largest score)
#pragma unroll
        for (int v = 0; v < V; ++v) c[v] *= part;
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (BIAS) c[v] += bias[v];
        if (!(l[v] > -INFINITY) || !(c[v] > -INFINITY)) c[v] = -INFINITY;
        if (two && v * 32 + lane < p.E) values[v * 32 + lane] = c[v];
        if (!BIAS) c[v] = l[v];
        choice.key[v] = c[v] > -INFINITY ? order_key(c[v]) : 0u;
        if (GROUPS && !two && v * 32 + lane < p.E) values[v * 32 + lane] = c[v];
      }
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        choice.key[v] = l[v] > -INFINITY ? order_key(l[v]) : 0u;
        if (GROUPS && v * 32 + lane < p.E) values[v * 32 + lane] = l[v] > -INFINITY ? l[v] : -INFINITY;
      }
    }
    if constexpr (GROUPS) {
      __syncwarp();
      const int g = lane / parts;
      float one = -INFINITY, second = -INFINITY;
      if (g < p.groups)
        for (int i = lane & (parts - 1); i < p.group_experts; i += parts) {
          const float x = values[g * p.group_experts + i];
          second = fmaxf(second, fminf(one, x));
          one = fmaxf(one, x);
        }
      for (int i = parts >> 1; i > 0; i >>= 1) {
        const float a = __shfl_xor_sync(~0u, one, i), b = __shfl_xor_sync(~0u, second, i);
        second = fmaxf(fminf(one, a), fmaxf(second, b));
        one = fmaxf(one, a);
      }
      __syncwarp();
      const float value = two && second > -INFINITY ? one + second : one;
      // rounds of the best group, the first of equal ones; the lanes of a group go together
      bool open = g < p.groups && value > -INFINITY;
      const uint32_t key = open ? order_key(value) : 0u;
      uint32_t kept = 0, worst = 0;
      for (int i = 0; i < p.top_groups; ++i) {
        const uint32_t m = __reduce_max_sync(~0u, open ? key : 0u);
        if (m <= kDeadKey) break;
        const int at = (__ffs(__ballot_sync(~0u, open && key == m)) - 1) / parts;
        if (g == at) open = false;
        kept |= 1u << at;
        worst = m;
      }
      if (scores) {
        const uint32_t next = __reduce_max_sync(~0u, open ? key : 0u);
        if (next > kDeadKey) {  // (sums of two: twice the error, and roundings of values)
          const float a = key_value(worst), b = key_value(next);
          if (a - b <= 2.f * error + 0x1p-21f * (fabsf(a) + fabsf(b) + bias_size)) sure = false;
        }
      }
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (!(kept & group_bit[v])) choice.key[v] = 0;
    }
    int mine = -1;  // lane i: the i-th chosen
    if (sure) {
      // With a bias, values too close to tell: go on until one is clearly behind (what is behind that cannot be among the k), then by FP64
      bool close_ones = false;
      float last = INFINITY;
      int last_expert = -1, m = 0;
      for (;; ++m) {
        uint32_t key;
        int e;
        if (!BIAS && m == p.k) break;
        if (!choice.best(lane, key, e)) break;
        if (BIAS) {
          const float value = key_value(key);
          const bool near = m > 0 && last - value <= error + 0x1p-22f * (fabsf(value) + bias_size);
          if (m >= p.k && !near) break;
          if (m == 32) {  // (no end in sight)
            sure = false;
            break;
          }
          // (the same logit under the same bias: a tie, whatever the arithmetic)
          close_ones |= near && !(logit<T>(row, e) == logit<T>(row, last_expert) && p.bias[e] == p.bias[last_expert]);
          last = value;
          last_expert = e;
        }
        if (lane == m) mine = e;
        choice.take(lane, e);
      }
      if (BIAS && sure && close_ones) mine = order64<T, V>(p, row, top, lane, m, mine);
    }
    if (!sure) {
      choose64<T, V>(p, row, top, lane, chosen);
      mine = lane < p.k ? chosen[lane] : -1;
      __syncwarp();
    }
    if (lane >= p.k) mine = -1;
    // weights: lane i's
    float w = 0.f;
    const float lm = mine >= 0 ? logit<T>(row, mine) : -INFINITY;
    if (p.renorm) {
      // in proportion to exp(z), z = l or the logarithm of the sigmoid of l, which cannot underflow all together
      const float z = mine < 0 ? -INFINITY : (p.sigmoid ? fminf(lm, 0.f) - log1pf(expf(-fabsf(lm))) : lm);
      float zmax = z;
      asm volatile("redux.sync.max.f32 %0, %0, 0xffffffff;" : "+f"(zmax));
      const float u = mine < 0 ? 0.f : expf(z - zmax);
      w = p.scale * (u / warp_sum(u));
    } else if (mine >= 0) {
      w = p.scale * (p.sigmoid ? 1.f / (1.f + expf(-lm)) : expf(lm - top) * inv);
    }
    if (lane < p.k) {
      p.experts[t * p.k + lane] = mine;
      p.weights[t * p.k + lane] = mine < 0 ? 0.f : (nan ? __int_as_float(0x7fffffff) : w);
    }
  }
}

struct RouteBackwardParams {
  int64_t T, ld, ldd;
  int E, k, sigmoid, renorm;
  float scale;
  const void* logits;
  void* dlogits;
  const float* dweights;
  const int32_t* experts;
};

// One warp has a token, lane i its i-th slot; the row of gradients is put together in shared memory.
template <typename T, int V>
__global__ void __launch_bounds__(32 * kRouteWarps) route_backward_kernel(const RouteBackwardParams p) {
  extern __shared__ float rows[];  // E for each warp
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float* dl = rows + warp * p.E;
  wait_for_stream();
  for (int64_t t = (int64_t)blockIdx.x * kRouteWarps + warp; t < p.T; t += (int64_t)gridDim.x * kRouteWarps) {
    const T* row = static_cast<const T*>(p.logits) + t * p.ld;
    int e = lane < p.k ? p.experts[t * p.k + lane] : -1;
    if (e >= p.E) e = -1;
    const float g = e >= 0 ? p.scale * p.dweights[t * p.k + lane] : 0.f;
    const float lm = e >= 0 ? to_float(row[e]) : -INFINITY;
    const bool full = !p.renorm && !p.sigmoid;  // every expert has a gradient
    float l[V], top = -INFINITY, sum = 0.f;
    if (full) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const int i = v * 32 + lane;
        l[v] = i < p.E ? to_float(row[i]) : -INFINITY;
        top = fmaxf(top, l[v]);
      }
      asm volatile("redux.sync.max.f32 %0, %0, 0xffffffff;" : "+f"(top));
#pragma unroll
      for (int v = 0; v < V; ++v) {
        l[v] = l[v] == -INFINITY ? 0.f : expf(l[v] - top);
        sum += l[v];
      }
      sum = warp_sum(sum);
    }
    float d = 0.f, along = 0.f;
    if (p.renorm) {
      const float z = e < 0 ? -INFINITY : (p.sigmoid ? fminf(lm, 0.f) - log1pf(expf(-fabsf(lm))) : lm);
      float zmax = z;
      asm volatile("redux.sync.max.f32 %0, %0, 0xffffffff;" : "+f"(zmax));
      const float w = e < 0 ? 0.f : expf(z - zmax), all = warp_sum(w), u = e < 0 ? 0.f : w / all;
      d = u * (g - warp_sum(u * g));
      if (p.sigmoid) d *= 1.f / (1.f + expf(lm));
    } else if (p.sigmoid) {
      const float s = 1.f / (1.f + expf(-lm));
      d = e < 0 ? 0.f : g * s * (1.f / (1.f + expf(lm)));
    } else {
      const float s = e < 0 ? 0.f : expf(lm - top) / sum;
      along = warp_sum(s * g);
      d = g;
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (v * 32 + lane < p.E) dl[v * 32 + lane] = 0.f;
    const uint32_t same = __match_any_sync(~0u, e);
    if (__any_sync(~0u, e >= 0 && (same & (same - 1)))) {  // an expert twice: one after the other
      for (int i = 0; i < p.k; ++i) {
        if (lane == i && e >= 0) dl[e] += d;
        __syncwarp();
      }
    } else {
      __syncwarp();
      if (e >= 0) dl[e] = d;
    }
    __syncwarp();
    T* out = static_cast<T*>(p.dlogits) + t * p.ldd;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int i = v * 32 + lane;
      if (i < p.E) out[i] = round_to<T>(full ? (sum > 0.f || sum != sum ? l[v] / sum * (dl[i] - along) : 0.f) : dl[i]);
    }
    __syncwarp();
  }
}

// f(number of experts that a lane has, as a type)
template <typename F>
sp24_status with_experts(int64_t E, F&& f) {
  if (E <= 32) return f(std::integral_constant<int, 1>{});
  if (E <= 64) return f(std::integral_constant<int, 2>{});
  if (E <= 128) return f(std::integral_constant<int, 4>{});
  if (E <= 256) return f(std::integral_constant<int, 8>{});
  if (E <= 512) return f(std::integral_constant<int, 16>{});
  return f(std::integral_constant<int, 32>{});
}

// blocks of a warp to a token, at most `per_sm` to an SM
unsigned route_blocks(int64_t T, int per_sm) {
  const int64_t blocks = (T + kRouteWarps - 1) / kRouteWarps, most = (int64_t)sm_count() * per_sm;
  return (unsigned)(blocks < most ? blocks : most);
}

}  // namespace
}  // namespace sp24

using namespace sp24;

extern "C" sp24_status sp24_route(sp24_dtype t, int64_t T, int64_t E, const void* logits, int64_t ld, sp24_score score, const float* bias,
                                  int groups, int top_groups, sp24_group_score group_score, int k, int renorm, float scale, float* weights,
                                  int32_t* experts, void* stream) {
  SP24_RETURN_IF(!is_float_type(t), SP24_ERR_DTYPE);
  SP24_RETURN_IF(T < 0 || T > (int64_t(1) << 40) || E < 1 || E > kMostExperts, SP24_ERR_SHAPE);
  SP24_RETURN_IF(groups < 1 || groups > kMostGroups || E % groups || top_groups < 1 || top_groups > groups, SP24_ERR_SHAPE);
  SP24_RETURN_IF(k < 1 || k > kMostChosen || k > top_groups * (E / groups), SP24_ERR_SHAPE);
  SP24_RETURN_IF((score != SP24_SCORE_SOFTMAX && score != SP24_SCORE_SIGMOID) || (group_score != SP24_GROUP_MAX && group_score != SP24_GROUP_TOP2),
                 SP24_ERR_UNSUPPORTED);
  if (T == 0) return SP24_OK;
  SP24_RETURN_IF(logits == nullptr || weights == nullptr || experts == nullptr, SP24_ERR_NULL);
  SP24_RETURN_IF(!row_fits(T, E, ld), SP24_ERR_STRIDE);
  SP24_RETURN_IF(!aligned(logits, elem_bytes(t)) || !aligned(bias, 4) || !aligned(weights, 4) || !aligned(experts, 4), SP24_ERR_ALIGN);
  const sp24_status arch = check_arch();
  SP24_RETURN_IF(arch != SP24_OK, arch);
  RouteParams p = {};
  p.T = T; p.ld = ld; p.E = (int)E; p.k = k;
  p.groups = groups; p.group_experts = (int)(E / groups); p.top_groups = top_groups;
  p.sigmoid = score == SP24_SCORE_SIGMOID; p.top2 = group_score == SP24_GROUP_TOP2 && p.group_experts > 1 ? 1 : 0;
  p.renorm = renorm != 0; p.scale = scale;
  p.logits = logits; p.bias = bias; p.weights = weights; p.experts = experts;
  return with_float_type(t, [&](auto type) {
    using Type = typename decltype(type)::type;
    return with_experts(E, [&](auto v) {
      return with_flags([&](auto with_bias, auto with_groups) {
        return launch_overlapped(route_kernel<Type, decltype(v)::value, decltype(with_bias)::value, decltype(with_groups)::value>, dim3(route_blocks(T, 4)),
                                 dim3(32 * kRouteWarps), decltype(with_groups)::value ? (size_t)(kRouteWarps * E * 4) : 0, static_cast<cudaStream_t>(stream), 1, p);
      }, bias != nullptr, groups > 1);
    });
  });
}

extern "C" sp24_status sp24_route_backward(sp24_dtype t, int64_t T, int64_t E, const float* dweights, const void* logits, int64_t ld,
                                           const int32_t* experts, int k, sp24_score score, int renorm, float scale, void* dlogits, int64_t ldd,
                                           void* stream) {
  SP24_RETURN_IF(!is_float_type(t), SP24_ERR_DTYPE);
  SP24_RETURN_IF(T < 0 || T > (int64_t(1) << 40) || E < 1 || E > kMostExperts || k < 1 || k > kMostChosen, SP24_ERR_SHAPE);
  SP24_RETURN_IF(score != SP24_SCORE_SOFTMAX && score != SP24_SCORE_SIGMOID, SP24_ERR_UNSUPPORTED);
  if (T == 0) return SP24_OK;
  SP24_RETURN_IF(dweights == nullptr || logits == nullptr || experts == nullptr || dlogits == nullptr, SP24_ERR_NULL);
  SP24_RETURN_IF(!row_fits(T, E, ld) || !row_fits(T, E, ldd), SP24_ERR_STRIDE);
  SP24_RETURN_IF(dlogits == logits && T > 1 && ld != ldd, SP24_ERR_STRIDE);
  SP24_RETURN_IF(!aligned(logits, elem_bytes(t)) || !aligned(dlogits, elem_bytes(t)) || !aligned(dweights, 4) || !aligned(experts, 4), SP24_ERR_ALIGN);
  const sp24_status arch = check_arch();
  SP24_RETURN_IF(arch != SP24_OK, arch);
  RouteBackwardParams p = {};
  p.T = T; p.ld = ld; p.ldd = ldd; p.E = (int)E; p.k = k;
  p.sigmoid = score == SP24_SCORE_SIGMOID; p.renorm = renorm != 0; p.scale = scale;
  p.logits = logits; p.dlogits = dlogits; p.dweights = dweights; p.experts = experts;
  return with_float_type(t, [&](auto type) {
    using Type = typename decltype(type)::type;
    return with_experts(E, [&](auto v) {
      return launch_overlapped(route_backward_kernel<Type, decltype(v)::value>, dim3(route_blocks(T, 8)), dim3(32 * kRouteWarps),
                               (size_t)(kRouteWarps * E * 4), static_cast<cudaStream_t>(stream), 1, p);
    });
  });
}
