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
  float scale, score_error;
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
// The choice is k rounds of the largest key, the lowest index first.  FP64 where FP32 does not tell: a score is off by at most 2^-22 of
// it (sigmoid: the exponential's two units in the last place, a sum, a division) or 2^-18 (softmax: the difference to the largest
// logit, up to 88 where the score is not 0, is rounded before the exponential), s + b by half a step more.
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

template <typename T, int V>
__global__ void __launch_bounds__(32 * kRouteWarps) route_kernel(const RouteParams p) {
  __shared__ int32_t chosen_of[kRouteWarps][kMostChosen];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int32_t* chosen = chosen_of[warp];
  wait_for_stream();
  for (int64_t t = (int64_t)blockIdx.x * kRouteWarps + warp; t < p.T; t += (int64_t)gridDim.x * kRouteWarps) {
    const void* row = static_cast<const T*>(p.logits) + t * p.ld;
    float l[V];
    float top = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int e = v * 32 + lane;
      l[v] = e < p.E ? logit<T>(row, e) : -INFINITY;
      nan |= l[v] != l[v];
      top = fmaxf(top, l[v]);
    }
    asm volatile("redux.sync.max.f32 %0, %0, 0xffffffff;" : "+f"(top));
    nan = __any_sync(~0u, nan) || (!p.sigmoid && top == INFINITY);
    const bool scores = p.bias || (p.groups > 1 && p.top2), total = !p.sigmoid && !p.renorm;
    float sum = 1.f;
    Choice<V> choice;
    float by_group[V];  // SP24_GROUP_TOP2: s + bias
    float scored[V];
    if (scores || total) {
      float part = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        scored[v] = p.sigmoid ? 1.f / (1.f + expf(-l[v])) : (l[v] > -INFINITY ? expf(l[v] - top) : 0.f);
        part += scored[v];
      }
      if (!p.sigmoid) sum = warp_sum(part);
    }
    const float inv = 1.f / sum;
    bool sure = true;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int e = v * 32 + lane;
      float c = l[v];
      if (scores) {
        const float s = scored[v] * inv + (p.bias && e < p.E ? p.bias[e] : 0.f);
        by_group[v] = l[v] > -INFINITY && s > -INFINITY ? s : -INFINITY;
        if (p.bias) c = by_group[v];
      }
      choice.key[v] = c > -INFINITY ? order_key(c) : 0u;
    }
    if (p.groups > 1) {
      float mine = -INFINITY, error = 0.f;  // of group `lane`: its value, and how far it may be off
      for (int g = 0; g < p.groups; ++g) {
        const int first = g * p.group_experts, last = first + p.group_experts;
        uint32_t one = 0, two = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const int e = v * 32 + lane;
          const uint32_t x = e >= first && e < last ? (p.top2 ? (by_group[v] > -INFINITY ? order_key(by_group[v]) : 0u) : choice.key[v]) : 0u;
          two = max(two, min(one, x));
          one = max(one, x);
        }
        const uint32_t best = __reduce_max_sync(~0u, one);
        float value = best > kDeadKey ? key_value(best) : -INFINITY;
        if (p.top2 && best > kDeadKey) {
          const uint32_t holders = __ballot_sync(~0u, one == best);
          if (lane == __ffs(holders) - 1) one = two;
          const uint32_t second = __reduce_max_sync(~0u, one);
          if (second > kDeadKey) value += key_value(second);
        }
        if (lane == g) mine = value;
      }
      if (scores) error = 2.f * p.score_error + 0x1p-21f * fabsf(mine);  // (of two scores, each at most 1)
      bool open = lane < p.groups, kept = false;
      float worst = INFINITY, slack = 0.f;
      for (int i = 0; i < p.top_groups; ++i) {
        const uint32_t m = __reduce_max_sync(~0u, open && mine > -INFINITY ? order_key(mine) : 0u);
        if (m <= kDeadKey) break;
        const int at = __ffs(__ballot_sync(~0u, open && mine > -INFINITY && order_key(mine) == m)) - 1;
        if (lane == at) { open = false; kept = true; }
        worst = key_value(m);
        slack = __shfl_sync(~0u, error, at);
      }
      if (scores && __any_sync(~0u, open && mine > -INFINITY && mine + error + slack >= worst)) sure = false;
      const uint32_t groups = __ballot_sync(~0u, kept);
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (!(groups >> ((v * 32 + lane) / p.group_experts & 31) & 1)) choice.key[v] = 0;
    }
    // k rounds, and with a bias one more: the best that is left has to be as clearly behind as the others behind one another
    float last = INFINITY, last_l = 0.f, last_b = 0.f, last_s = 0.f;
    const int rounds = p.bias && p.k < p.E ? p.k + 1 : p.k;
    int mine = -1;  // lane i: the i-th chosen
    if (sure) {
      for (int i = 0; i < rounds; ++i) {
        uint32_t key;
        int e;
        if (!choice.best(lane, key, e)) break;
        if (p.bias) {
          const float v = key_value(key), li = logit<T>(row, e), b = p.bias[e], s = fabsf(v - b);
          const float error = p.score_error * (s + last_s) + 0x1p-22f * (fabsf(v) + fabsf(b) + fabsf(last_b));
          if (i && last - v <= error && !(li == last_l && b == last_b)) sure = false;
          last = v;
          last_l = li;
          last_b = b;
          last_s = s;
        }
        if (i == p.k) break;
        if (lane == i) mine = e;
        choice.take(lane, e);
      }
    }
    if (!sure) {
      choose64<T, V>(p, row, top, lane, chosen);
      mine = lane < p.k ? chosen[lane] : -1;
      __syncwarp();
    }
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
    for (int i = lane; i < p.E; i += 32) dl[i] = 0.f;
    __syncwarp();
    for (int i = 0; i < p.k; ++i) {  // (the same expert twice: one after the other)
      if (lane == i && e >= 0) dl[e] += d;
      __syncwarp();
    }
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
  return f(std::integral_constant<int, 32>{});
}

unsigned route_blocks(int64_t T) {
  const int64_t blocks = (T + kRouteWarps - 1) / kRouteWarps, most = (int64_t)sm_count() * 64;
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
  p.renorm = renorm != 0; p.scale = scale; p.score_error = p.sigmoid ? 0x1p-22f : 0x1p-18f;
  p.logits = logits; p.bias = bias; p.weights = weights; p.experts = experts;
  return with_float_type(t, [&](auto type) {
    using Type = typename decltype(type)::type;
    return with_experts(E, [&](auto v) {
      return launch_overlapped(route_kernel<Type, decltype(v)::value>, dim3(route_blocks(T)), dim3(32 * kRouteWarps), 0, static_cast<cudaStream_t>(stream), 1, p);
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
      return launch_overlapped(route_backward_kernel<Type, decltype(v)::value>, dim3(route_blocks(T)), dim3(32 * kRouteWarps),
                               (size_t)(kRouteWarps * E * 4), static_cast<cudaStream_t>(stream), 1, p);
    });
  });
}
