// Routing of tokens to experts, and its gradient.
#include <cfloat>

#include "sp24_rows.cuh"

namespace sp24 {
namespace {

constexpr int kMostGroups = 32;
constexpr int kRouteWarps = 8;

struct RouteParams {
  int64_t T, ld;
  int E, k, groups, group_experts, top_groups;
  int group_parts, group_stride;  // lanes that look for the best of a group (a power of two), and how far apart the groups lie in shared memory
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

// The whole choice under a bias in FP64, for the tokens of which FP32 cannot tell it: rare, so kept out of the way.
template <typename T, int V>
__device__ __noinline__ void choose64(const RouteParams& p, const void* row, float top_logit, int lane, int32_t* chosen) {
  double c[V];
  double sum = 0.0;
  for (int v = 0; v < V; ++v) {
    const int e = v * 32 + lane;
    const float l = e < p.E ? logit<T>(row, e) : -INFINITY;
    c[v] = !(l > -INFINITY) ? -INFINITY : p.sigmoid ? 1.0 / (1.0 + exp(-(double)l)) : exp((double)l - (double)top_logit);  // (NaN too)
    if (l > -INFINITY) sum += c[v];
  }
  sum = p.sigmoid ? 1.0 : warp_sum(sum);
  for (int v = 0; v < V; ++v) {
    const int e = v * 32 + lane;
    if (!(c[v] > -INFINITY)) continue;
    c[v] = c[v] / sum + (double)p.bias[e];
    if (!(c[v] > -INFINITY)) c[v] = -INFINITY;
  }
  if (p.groups > 1) {
    double mine = -INFINITY;  // of group `lane`
    for (int g = 0; g < p.groups; ++g) {
      double one = -INFINITY, two = -INFINITY;
      for (int v = 0; v < V; ++v) {
        const int e = v * 32 + lane;
        if (e / p.group_experts == g && e < p.E) {
          two = fmax(two, fmin(one, c[v]));
          one = fmax(one, c[v]);
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

// The groups that stay, by FP64: lane (group, part) has every so manieth expert of its group.
template <typename T>
__device__ __noinline__ uint32_t groups64(const RouteParams& p, const void* row, float top_logit, int lane) {
  const int parts = p.group_parts, g = lane / parts, first = g * p.group_experts;
  const bool mine = g < p.groups;
  auto score = [&](int i) {
    const double l = (double)logit<T>(row, first + i);
    return !(l > -INFINITY) ? -INFINITY : p.sigmoid ? 1.0 / (1.0 + exp(-l)) : exp(l - (double)top_logit);
  };
  double sum = 0.0, one = -INFINITY, two = -INFINITY;
  if (!p.sigmoid) {
    if (mine)
      for (int i = lane & (parts - 1); i < p.group_experts; i += parts) sum += fmax(score(i), 0.0);
    sum = warp_sum(sum);
  }
  if (mine)
    for (int i = lane & (parts - 1); i < p.group_experts; i += parts) {
      double x = score(i);
      if (x > -INFINITY) x = (p.sigmoid ? x : x / sum) + (p.bias ? (double)p.bias[first + i] : 0.0);
      if (!(x > -INFINITY)) continue;
      two = fmax(two, fmin(one, x));
      one = fmax(one, x);
    }
  for (int i = parts >> 1; i > 0; i >>= 1) {
    const double a = __shfl_xor_sync(~0u, one, i), b = __shfl_xor_sync(~0u, two, i);
    two = fmax(fmin(one, a), fmax(two, b));
    one = fmax(one, a);
  }
  const double value = p.top2 && two > -INFINITY ? one + two : one;
  int place = 0;
  for (int h = 0; h < p.groups; ++h) {
    const double other = __shfl_sync(~0u, value, h * parts);
    place += other > value || (other == value && h < g);
  }
  const uint32_t lanes = __ballot_sync(~0u, mine && (lane & (parts - 1)) == 0 && place < p.top_groups);
  uint32_t kept = 0;
  for (int h = 0; h < p.groups; ++h) kept |= (lanes >> (h * parts) & 1) << h;
  return kept;
}

// What a lane keeps of its experts over the tokens.
template <int V>
struct LaneExperts {
  float bias[V], bias_size;  // the largest finite |bias| of all
  uint8_t group_of[V];
  __device__ __forceinline__ LaneExperts(const RouteParams& p, int lane, bool with_bias, bool with_groups) {
    bias_size = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int e = v * 32 + lane;
      if (with_bias) {
        bias[v] = e < p.E ? p.bias[e] : -INFINITY;
        bias_size = fmaxf(bias_size, fabsf(bias[v]) < INFINITY ? fabsf(bias[v]) : 0.f);
      }
      if (with_groups) group_of[v] = e < p.E ? e / p.group_experts : 0;
    }
    if (with_bias) asm volatile("redux.sync.max.f32 %0, %0, 0xffffffff;" : "+f"(bias_size));
  }
};

// One token, by a warp: any number of experts and groups, any alignment.  Scores for the choice come from the special-function units; the weights are computed again, exactly,
// for the chosen.  `values`: room for a row for each group.
template <typename T, int V, bool BIAS, bool GROUPS>
__device__ __forceinline__ void route_token(const RouteParams& p, int64_t t, int lane, const LaneExperts<V>& x, uint2* mine_of, int32_t* chosen, float* values) {
  const bool two = GROUPS && p.top2, scores = BIAS || two, total = !p.sigmoid && !p.renorm;
  const int parts = p.group_parts, pad = p.group_stride - p.group_experts;
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
      if (BIAS) c[v] += x.bias[v];
      if (!(l[v] > -INFINITY) || !(c[v] > -INFINITY)) c[v] = -INFINITY;
      if (two && v * 32 + lane < p.E) values[v * 32 + lane + x.group_of[v] * pad] = c[v];
      if (!BIAS) c[v] = l[v];
      choice.key[v] = c[v] > -INFINITY ? order_key(c[v]) : 0u;
      if (GROUPS && !two && v * 32 + lane < p.E) values[v * 32 + lane + x.group_of[v] * pad] = c[v];
    }
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) {
      choice.key[v] = l[v] > -INFINITY ? order_key(l[v]) : 0u;
      if (GROUPS && v * 32 + lane < p.E) values[v * 32 + lane + x.group_of[v] * pad] = l[v] > -INFINITY ? l[v] : -INFINITY;
    }
  }
  if constexpr (GROUPS) {
    __syncwarp();
    const int g = lane / parts;
    float one = -INFINITY, second = -INFINITY;
    if (g < p.groups)
      for (int i = lane & (parts - 1); i < p.group_experts; i += parts) {
        const float y = values[g * p.group_stride + i];
        second = fmaxf(second, fminf(one, y));
        one = fmaxf(one, y);
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
        if (a - b <= 2.f * error + 0x1p-21f * (fabsf(a) + fabsf(b) + x.bias_size)) kept = groups64<T>(p, row, top, lane);
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (!(kept >> x.group_of[v] & 1)) choice.key[v] = 0;
  }
  int mine = -1;  // lane i: the i-th chosen
  // The k-th largest of the lanes' largest (k rounds, equal ones of several lanes in one) is not above the k-th largest of all: what reaches it, less what
  // FP32 may be off, are the candidates, hardly more than k of them.  Each is in a lane's hands then, and its place is the number of those before it.
  int candidates = 0;
  float near = 0.f;  // (with a bias: how far apart two values must be to be told apart)
  uint32_t m = choice.key[0];
#pragma unroll
  for (int v = 1; v < V; ++v) m = max(m, choice.key[v]);
  uint32_t least = 0;
  for (int i = 0; i < p.k; ++i) {
    const uint32_t top_key = __reduce_max_sync(~0u, m);
    if (top_key <= kDeadKey) { least = 0; break; }
    least = top_key;
    if (m == top_key) m = 0;
  }
  if (BIAS) {
    near = error + 0x1p-22f * (2.f + 2.f * x.bias_size);  // (sums of a score, at most 1, and a bias; rounded by half a step of theirs)
    if (least) least = order_key(key_value(least) - near);
  }
  least = max(least, kDeadKey + 1);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const bool in = choice.key[v] >= least;
    const uint32_t all = __ballot_sync(~0u, in);
    const int at = candidates + __popc(all & ((1u << lane) - 1));
    if (in && at < 32) mine_of[at] = make_uint2(choice.key[v], v * 32 + lane);
    candidates += __popc(all);
  }
  __syncwarp();
  if (candidates <= 32) {
    const uint2 own = lane < candidates ? mine_of[lane] : make_uint2(0, 0);
    int place = lane < candidates ? 0 : 32;
    for (int i = 0; i < candidates; ++i) {
      const uint2 other = mine_of[i];  // (the same for all lanes)
      place += other.x > own.x || (other.x == own.x && other.y < own.y);
    }
    __syncwarp();
    if (lane < candidates) mine_of[place] = own;
    __syncwarp();
    const uint2 here = lane < candidates ? mine_of[lane] : make_uint2(0, 0);
    mine = lane < candidates ? (int)here.y : -1;
    if (BIAS) {
      // A chosen one against the one before, all that are left against the last chosen: there may be equals of it before one that it is too close to.
      const uint2 before = lane > 0 && lane < candidates ? mine_of[min(lane, p.k) - 1] : make_uint2(0, 0);
      bool doubt = lane > 0 && lane < candidates && key_value(before.x) - key_value(here.x) <= near;
      // (the same logit under the same bias: a tie, whatever the arithmetic)
      if (doubt) doubt = !(logit<T>(row, here.y) == logit<T>(row, before.y) && p.bias[here.y] == p.bias[before.y]);
      if (__any_sync(~0u, doubt)) mine = order64<T, V>(p, row, top, lane, candidates, mine);
    }
    __syncwarp();
  } else if constexpr (BIAS) {
    choose64<T, V>(p, row, top, lane, chosen);
    mine = lane < p.k ? chosen[lane] : -1;
    __syncwarp();
  } else {  // many equal logits, or a large k: one after the other
    for (int i = 0; i < p.k; ++i) {
      uint32_t key;
      int e;
      if (!choice.best(lane, key, e)) break;
      if (lane == i) mine = e;
      choice.take(lane, e);
    }
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
    w = p.scale * __fdividef(u, warp_sum(u));
  } else if (mine >= 0) {
    w = p.scale * (p.sigmoid ? 1.f / (1.f + expf(-lm)) : expf(lm - top) * inv);
  }
  if (lane < p.k) {
    p.experts[t * p.k + lane] = mine;
    p.weights[t * p.k + lane] = mine < 0 ? 0.f : (nan ? __int_as_float(0x7fffffff) : w);
  }
}

template <int V>
constexpr int kRouteBlocks = V <= 8 ? 3 : 1;  // to an SM

template <typename T, int V, bool BIAS, bool GROUPS>
__global__ void __launch_bounds__(32 * kRouteWarps) route_kernel(const RouteParams p) {
  __shared__ int32_t chosen_of[kRouteWarps][kMostChosen];
  __shared__ uint2 candidates_of[kRouteWarps][32];  // key, expert
  extern __shared__ float values_of[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  wait_for_stream();
  const LaneExperts<V> x(p, lane, BIAS, GROUPS);
  for (int64_t t = (int64_t)blockIdx.x * kRouteWarps + warp; t < p.T; t += (int64_t)gridDim.x * kRouteWarps)
    route_token<T, V, BIAS, GROUPS>(p, t, lane, x, candidates_of[warp], chosen_of[warp], values_of + warp * p.groups * p.group_stride);
}

// ---- up to 256 experts in chunks: a token to eight lanes -----------------------------------------------------------
// Of a warp's 1600 instructions for a token of 256 experts with groups and a bias most are reductions over the warp and bookkeeping, which four tokens to a warp
// share: 460 a token.  What bounds it then is latency, of which 96 registers leave little to overlap: five blocks to an SM, 740 at a time, for 1024 of 16384 tokens;
// 38 % of the issue slots are used.  Lane j of a token has the j-th eighth of its experts, whole 16-byte vectors; a group is 8 / groups lanes.  The k rounds: the largest of the
// lanes' largest; its lane finds it in shared memory, where it has the largest of each eight of its values to look under.  Tokens that FP32 does not decide, or with a NaN
// or +infinity among their logits, are done again by the whole warp (route_token).
// Us, device, 16384 tokens of 256 experts, a warp to a token and this: the 8 best, softmax 13.5, 11.1; of 8 groups, 4 stay, 26, 12.1; by sigmoid and bias, groups by the two
// best, 37, 16.4 (HBM: 2.9; of the 16, 7.4 are what the largest of a row takes, eight rounds of choosing 3.7, the scores 2, what is too close to tell 2).
constexpr int kChunkWarps = 4, kChunkTokens = 4 * kChunkWarps;
template <int V>
constexpr int kChunkRow = V + 4;  // floats of a lane's row in shared memory: lanes that read vectors together are in banks of their own

__device__ __forceinline__ float max_nan(float a, float b) {
  asm("max.NaN.f32 %0, %0, %1;" : "+f"(a) : "f"(b));
  return a;
}

template <typename T, bool BIAS, bool GROUPS>
__device__ __noinline__ void route_again(const RouteParams& p, int64_t t, int lane, uint2* mine_of, int32_t* chosen, float* values) {
  const LaneExperts<8> x(p, lane, BIAS, GROUPS);
  route_token<T, 8, BIAS, GROUPS>(p, t, lane, x, mine_of, chosen, values);
}

// s + b of one expert in FP64 (sigmoid)
template <typename T>
__device__ __noinline__ double exact_sigmoid(const RouteParams& p, const T* row, int e) {
  return 1.0 / (1.0 + exp(-(double)to_float(row[e]))) + (p.bias ? (double)p.bias[e] : 0.0);
}

// Whether the lane's group stays, by FP64: the sum of the two largest of the group's `n` candidates in this lane (places in the lane's chunk) and its other lanes'.
template <typename T>
__device__ __noinline__ bool exact_group(const RouteParams& p, const T* row, int lane, const float* places, int n) {
  const int j = lane & 7, chunk = p.E / 8, lanes = 8 / p.groups;
  double one = -INFINITY, two = -INFINITY;
  const int most = __reduce_max_sync(~0u, n);
  for (int i = 0; i < most; ++i) {
    const double x = i < n ? exact_sigmoid(p, row, j * chunk + __float_as_int(places[i])) : -INFINITY;
    two = fmax(two, fmin(one, x));
    one = fmax(one, x);
  }
  for (int i = 1; i < lanes; i <<= 1) {
    const double a = __shfl_xor_sync(~0u, one, i), b = __shfl_xor_sync(~0u, two, i);
    two = fmax(fmin(one, a), fmax(two, b));
    one = fmax(one, a);
  }
  const double value = two > -INFINITY ? one + two : one;
  int before = 0;
  for (int i = lanes; i < 8; i += lanes) {
    const double other = __shfl_xor_sync(~0u, value, i);
    before += other > value || (other == value && (j ^ i) < j);
  }
  return before < p.top_groups;
}

template <typename T, int V, bool BIAS, bool GROUPS>
__global__ void __launch_bounds__(32 * kChunkWarps) route_chunks_kernel(const RouteParams p) {
  constexpr int R = kChunkRow<V>, S = V / 8, N = 16 / sizeof(T);
  __shared__ __align__(16) float rows_of[kChunkWarps][32 * R];
  __shared__ __align__(16) float bias_rows[BIAS ? 8 * R : 4];
  __shared__ int32_t chosen_of[kChunkWarps][kMostChosen];
  __shared__ uint2 candidates_of[kChunkWarps][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, j = lane & 7;
  const int chunk = p.E / 8;
  const bool two = GROUPS && p.top2, scores = BIAS || two, total = !p.sigmoid && !p.renorm;
  wait_for_stream();
  float bias_size = 0.f;  // the largest finite |bias|
  if (BIAS) {
    __shared__ int size_bits;
    if (threadIdx.x == 0) size_bits = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < 8 * V; i += blockDim.x) {
      const float b = i % V < chunk ? p.bias[i / V * chunk + i % V] : -INFINITY;
      bias_rows[i / V * R + i % V] = b;
      if (fabsf(b) < INFINITY) bias_size = fmaxf(bias_size, fabsf(b));
    }
    atomicMax(&size_bits, __float_as_int(bias_size));
    __syncthreads();
    bias_size = __int_as_float(size_bits);
  }
  const int64_t t = ((int64_t)blockIdx.x * kChunkWarps + warp) * 4 + (lane >> 3);
  const bool live = t < p.T;
  const T* row = static_cast<const T*>(p.logits) + (live ? t : 0) * p.ld;
  float l[V];
#pragma unroll
  for (int v = 0; v < V; v += N) {
    Pairs<T> f = {};
    if (v < chunk && live) unpack<T>(*reinterpret_cast<const uint4*>(row + j * chunk + v), f);
#pragma unroll
    for (int n = 0; n < N / 2; ++n) {
      l[v + 2 * n] = v < chunk && live ? f[n].x : -INFINITY;
      l[v + 2 * n + 1] = v < chunk && live ? f[n].y : -INFINITY;
    }
  }
  auto over_token = [&](float v, auto op) {
#pragma unroll
    for (int i = 1; i < 8; i <<= 1) v = op(v, __shfl_xor_sync(~0u, v, i));
    return v;
  };
  auto larger = [](float a, float b) { return fmaxf(a, b); };
  auto sum_of = [](float a, float b) { return a + b; };
  float top = l[0];
#pragma unroll
  for (int v = 1; v < V; ++v) top = max_nan(top, l[v]);
  top = over_token(top, max_nan);
  bool again = !(top < INFINITY);
  const float base = fmaxf(top, -FLT_MAX);  // (nothing but -infinity: exponentials of 0)
  float error = 0.f, near = 0.f, inv = 1.f;
  float c[V];
  if (scores || total) {
    if (p.sigmoid) {
      error = 2.f * 1.5f * 0x1p-22f;  // (as in route_token)
    } else {
      float sum = 0.f;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        c[v] = exp2_fast(kLog2e * (l[v] - base));
        sum += c[v];
      }
      inv = 1.f / over_token(sum, sum_of);
      error = 2.f * 0x1p-20f * inv;
#pragma unroll
      for (int v = 0; v < V; ++v) c[v] *= inv;
    }
  }
  if (scores) {
    // (0 * l is 0 but for what may not be chosen, and NaN there)
#pragma unroll
    for (int v = 0; v < V; v += 4) {
      float4 b = make_float4(0.f, 0.f, 0.f, 0.f);
      if (BIAS) b = *reinterpret_cast<const float4*>(bias_rows + j * R + v);
      const float add[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int n = 0; n < 4; ++n) {
        if (p.sigmoid) c[v + n] = reciprocal_fast(1.f + exp2_fast(-kLog2e * l[v + n]));
        c[v + n] = fmaxf(c[v + n] + fmaf(l[v + n], 0.f, add[n]), -INFINITY);
      }
    }
    near = error + 0x1p-22f * (2.f + 2.f * bias_size);
  }
  bool kept = true;
  if constexpr (GROUPS) {
    const int lanes = 8 / p.groups;
    float one = -INFINITY, second = -INFINITY;
    if (two) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        second = fmaxf(second, fminf(one, c[v]));
        one = fmaxf(one, c[v]);
      }
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) one = fmaxf(one, BIAS ? c[v] : l[v]);
    }
    for (int i = 1; i < lanes; i <<= 1) {
      const float a = __shfl_xor_sync(~0u, one, i), b = __shfl_xor_sync(~0u, second, i);
      second = fmaxf(fminf(one, a), fmaxf(second, b));
      one = fmaxf(one, a);
    }
    const float value = two && second > -INFINITY ? one + second : one;
    int before = 0;
    for (int i = lanes; i < 8; i += lanes) {
      const float other = __shfl_xor_sync(~0u, value, i);
      before += other > value || (other == value && (j ^ i) < j);
    }
    kept = before < p.top_groups;
    if (scores && p.top_groups < p.groups) {
      const float worst = -over_token(kept ? -value : -INFINITY, larger), next = over_token(kept ? -INFINITY : value, larger);
      const bool doubt = next > -INFINITY && worst - next <= 2.f * error + 0x1p-21f * (4.f + 4.f * bias_size);
      if (!(two && p.sigmoid)) {
        again |= doubt;
      } else if (__any_sync(~0u, doubt && !again)) {
        // once more in FP64, with what is not clearly behind the second of the group
        int n = 0;
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (doubt && c[v] > -INFINITY && !(c[v] < second - near)) rows_of[warp][lane * R + n++] = __int_as_float(v);
        const bool exact = exact_group(p, row, lane, rows_of[warp] + lane * R, n);
        if (doubt) kept = exact;
      }
    }
  }
  // what is chosen by, in shared memory, and the largest of each eight of a lane's
  float* mine = rows_of[warp] + lane * R;
  float best[S];
#pragma unroll
  for (int v = 0; v < V; ++v)
    if (!BIAS) c[v] = l[v];
#pragma unroll
  for (int v = 0; v < V; v += 4) *reinterpret_cast<float4*>(mine + v) = make_float4(c[v], c[v + 1], c[v + 2], c[v + 3]);
  auto largest_of_eight = [](const float4& a, const float4& b) { return fmaxf(fmaxf(fmaxf(a.x, a.y), fmaxf(a.z, a.w)), fmaxf(fmaxf(b.x, b.y), fmaxf(b.z, b.w))); };
#pragma unroll
  for (int i = 0; i < S; ++i)
    best[i] = largest_of_eight(make_float4(c[8 * i], c[8 * i + 1], c[8 * i + 2], c[8 * i + 3]), make_float4(c[8 * i + 4], c[8 * i + 5], c[8 * i + 6], c[8 * i + 7]));
  auto largest = [&] {
    float m = best[0];
#pragma unroll
    for (int i = 1; i < S; ++i) m = fmaxf(m, best[i]);
    return m;
  };
  float lane_best = kept ? largest() : -INFINITY;
  int chosen = -1;  // lane i of the token: the i-th
  float last = INFINITY;
  int last_expert = 0;
  bool followed = false, open = BIAS;  // whether what comes next is clearly behind the k chosen is still to be seen: after ties it takes more than one round
  for (int i = 0; i < p.k || (BIAS && i < p.k + 8 && __any_sync(~0u, open)); ++i) {
    const float m = over_token(lane_best, larger);
    const uint32_t holders = __ballot_sync(~0u, lane_best == m) >> (lane & 24) & 0xffu;
    const int w = (lane & 24) + __ffs(holders) - 1;
    // where each lane's largest is: the first of the eight, the first in it
    int at = 0;
#pragma unroll
    for (int s = S - 1; s > 0; --s)
      if (best[s] == lane_best) at = s;
    if (best[0] == lane_best) at = 0;
    float4 a = *reinterpret_cast<const float4*>(mine + 8 * at), b = *reinterpret_cast<const float4*>(mine + 8 * at + 4);
    int n = 7;
    if (b.z == lane_best) n = 6;
    if (b.y == lane_best) n = 5;
    if (b.x == lane_best) n = 4;
    if (a.w == lane_best) n = 3;
    if (a.z == lane_best) n = 2;
    if (a.y == lane_best) n = 1;
    if (a.x == lane_best) n = 0;
    const int place = 8 * at + n;
    const int e = __shfl_sync(~0u, j * chunk + place, w);
    const bool some = m > -INFINITY;
    int put = e;
    if (lane == w && some) {
      mine[place] = -INFINITY;
      a = *reinterpret_cast<const float4*>(mine + 8 * at);
      b = *reinterpret_cast<const float4*>(mine + 8 * at + 4);
      const float rest = largest_of_eight(a, b);
#pragma unroll
      for (int s = 0; s < S; ++s)
        if (s == at) best[s] = rest;
      lane_best = largest();
    }
    if (BIAS && i > 0) {
      const bool close = some && last - m <= near && (i < p.k || open);
      bool doubt = false;
      if (__any_sync(~0u, close)) {
        // (the same logit under the same bias: a tie, whatever the arithmetic)
        doubt = close && !(to_float(row[e]) == to_float(row[last_expert]) && p.bias[e] == p.bias[last_expert]);
        if (p.sigmoid && __any_sync(~0u, doubt)) {  // the two in FP64, by the token's even and odd lanes
          const double mine = exact_sigmoid(p, row, j & 1 ? e : last_expert), other = __shfl_xor_sync(~0u, mine, 1);
          const double a = j & 1 ? other : mine, b = j & 1 ? mine : other;
          if (doubt && !followed && (b > a || (b == a && e < last_expert))) {
            if (j == i - 1) chosen = e;
            put = last_expert;
          }
          again |= doubt && followed;  // (the one before followed as closely: it is not between these two alone)
        } else {
          again |= doubt;
        }
      }
      followed = close;
      if (i >= p.k) open = close;
    }
    last = m;
    last_expert = put;
    if (j == i && i < p.k) chosen = some ? put : -1;
  }
  again |= open;
  // weights: lane i's
  const float lm = chosen >= 0 && live ? to_float(row[chosen]) : -INFINITY;
  float weight = 0.f;
  if (p.renorm) {
    const float z = chosen < 0 ? -INFINITY : (p.sigmoid ? fminf(lm, 0.f) - log1pf(expf(-fabsf(lm))) : lm);
    const float zmax = over_token(z, larger), u = chosen < 0 ? 0.f : expf(z - zmax);
    weight = p.scale * __fdividef(u, over_token(u, sum_of));
  } else {
    weight = p.scale * (p.sigmoid ? 1.f / (1.f + expf(-lm)) : expf(lm - base) * inv);
  }
  if (live && j < p.k) {
    p.experts[t * p.k + j] = chosen;
    p.weights[t * p.k + j] = chosen < 0 ? 0.f : weight;
  }
  uint32_t tokens = __ballot_sync(~0u, again && live) & 0x01010101u;
  __syncwarp();
  while (tokens) {
    const int first = __ffs(tokens) - 1;
    tokens &= tokens - 1;
    route_again<T, BIAS, GROUPS>(p, __shfl_sync(~0u, t, first), lane, candidates_of[warp], chosen_of[warp], rows_of[warp]);
    __syncwarp();
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

// The same for up to 256 experts in whole vectors and up to eight slots: a token to eight lanes, lane j with the j-th eighth of the experts and the j-th slot.
// (Us, device, bf16 16384 x 128, 4 slots, softmax over all: a warp to a token 8.0, this 5.2; HBM: 1.4.)
template <typename T, int V>
__global__ void __launch_bounds__(32 * kChunkWarps) route_backward_chunks_kernel(const RouteBackwardParams p) {
  constexpr int N = 16 / sizeof(T);
  const int lane = threadIdx.x & 31, j = lane & 7, chunk = p.E / 8;
  wait_for_stream();
  const int64_t t = ((int64_t)blockIdx.x * kChunkWarps + (threadIdx.x >> 5)) * 4 + (lane >> 3);
  const bool live = t < p.T, slot = live && j < p.k;
  const T* row = static_cast<const T*>(p.logits) + (live ? t : 0) * p.ld;
  const bool full = !p.renorm && !p.sigmoid;
  int e = slot ? p.experts[t * p.k + j] : -1;
  if (e >= p.E) e = -1;
  const float g = e >= 0 ? p.scale * p.dweights[t * p.k + j] : 0.f;
  auto over_token = [&](float v, auto op) {
#pragma unroll
    for (int i = 1; i < 8; i <<= 1) v = op(v, __shfl_xor_sync(~0u, v, i));
    return v;
  };
  auto larger = [](float a, float b) { return fmaxf(a, b); };
  auto sum_of = [](float a, float b) { return a + b; };
  float l[V], top = -INFINITY, inv = 0.f;
  if (full) {
#pragma unroll
    for (int v = 0; v < V; v += N) {
      Pairs<T> f = {};
      if (v < chunk && live) unpack<T>(*reinterpret_cast<const uint4*>(row + j * chunk + v), f);
#pragma unroll
      for (int n = 0; n < N / 2; ++n) {
        l[v + 2 * n] = v < chunk ? f[n].x : -INFINITY;
        l[v + 2 * n + 1] = v < chunk ? f[n].y : -INFINITY;
      }
    }
  }
  const float lm = e >= 0 ? to_float(row[e]) : -INFINITY;
  if (full) {
#pragma unroll
    for (int v = 0; v < V; ++v) top = fmaxf(top, l[v]);
    top = over_token(top, larger);
    const float base = fmaxf(top, -FLT_MAX);
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      l[v] = expf(l[v] - base);
      sum += l[v];
    }
    sum = over_token(sum, sum_of);
    inv = sum == 0.f ? 0.f : 1.f / sum;  // (nothing but -infinity: no gradient)
    top = base;
  }
  float d = 0.f, along = 0.f;
  if (p.renorm) {
    const float z = e < 0 ? -INFINITY : (p.sigmoid ? fminf(lm, 0.f) - log1pf(expf(-fabsf(lm))) : lm);
    const float zmax = over_token(z, larger), w = e < 0 ? 0.f : expf(z - zmax), all = over_token(w, sum_of), u = e < 0 ? 0.f : w / all;
    d = u * (g - over_token(u * g, sum_of));
    if (p.sigmoid) d *= 1.f / (1.f + expf(lm));
  } else if (p.sigmoid) {
    d = e < 0 ? 0.f : g * (1.f / (1.f + expf(-lm))) * (1.f / (1.f + expf(lm)));
  } else {
    along = over_token(e < 0 ? 0.f : expf(lm - top) * inv * g, sum_of);
    d = g;
  }
  float dl[V] = {};
  for (int i = 0; i < p.k; ++i) {
    const int at = __shfl_sync(~0u, e, (lane & 24) + i) - j * chunk;
    const float x = __shfl_sync(~0u, d, (lane & 24) + i);
    if (at >= 0 && at < chunk) {
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (v == at) dl[v] += x;
    }
  }
  if (full) {
#pragma unroll
    for (int v = 0; v < V; ++v) dl[v] = l[v] * inv * (dl[v] - along);
  }
  if (!live) return;
  T* out = static_cast<T*>(p.dlogits) + t * p.ldd + j * chunk;
#pragma unroll
  for (int v = 0; v < V; v += N) {
    Pairs<T> f;
#pragma unroll
    for (int n = 0; n < N / 2; ++n) f[n] = make_float2(dl[v + 2 * n], dl[v + 2 * n + 1]);
    if (v < chunk) *reinterpret_cast<uint4*>(out + v) = pack<T>(f);
  }
}

// whether an eighth of the experts is whole vectors, and there is a lane to each slot
bool whole_chunks(int64_t E, int64_t es, int k) { return E <= 256 && E % 8 == 0 && E / 8 * es % 16 == 0 && k <= 8; }

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
  const int64_t blocks = (T + kRouteWarps - 1) / kRouteWarps, most = (int64_t)sm_count() * per_sm, rounds = (blocks + most - 1) / most;
  return (unsigned)((blocks + rounds - 1) / rounds);
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
  p.group_parts = 1;
  while (2 * p.group_parts * groups <= 32) p.group_parts *= 2;
  // Each group's lanes in banks of their own, but for the few shapes (E above 780, groups of 34 to 44, 67 or 68) whose rows would ask for more than
  // the shared memory that a kernel has without an opt-in.
  p.group_stride = p.group_experts + ((p.group_parts - p.group_experts) & 31);
  constexpr size_t kStatic = kRouteWarps * (kMostChosen * sizeof(int32_t) + 32 * sizeof(uint2));  // (route_kernel's arrays)
  if (kRouteWarps * groups * p.group_stride * sizeof(float) + kStatic > 48 * 1024) p.group_stride = p.group_experts;
  p.sigmoid = score == SP24_SCORE_SIGMOID; p.top2 = group_score == SP24_GROUP_TOP2 && p.group_experts > 1 ? 1 : 0;
  p.renorm = renorm != 0; p.scale = scale;
  p.logits = logits; p.bias = bias; p.weights = weights; p.experts = experts;
  return with_float_type(t, [&](auto type) {
    using Type = typename decltype(type)::type;
    const bool chunks = whole_chunks(E, sizeof(Type), k) && groups <= 8 && 8 % groups == 0 && aligned16(logits) &&
                        (T == 1 || ld * (int64_t)sizeof(Type) % 16 == 0) && T < int64_t(1) << 35;
    if (chunks) {
      auto run = [&](auto v) {
        return with_flags([&](auto with_bias, auto with_groups) {
          return launch_overlapped(route_chunks_kernel<Type, decltype(v)::value, decltype(with_bias)::value, decltype(with_groups)::value>,
                                   dim3((unsigned)((T + kChunkTokens - 1) / kChunkTokens)), dim3(32 * kChunkWarps), 0, static_cast<cudaStream_t>(stream), 1, p);
        }, bias != nullptr, groups > 1);
      };
      if (E <= 64) return run(std::integral_constant<int, 8>{});
      if (E <= 128) return run(std::integral_constant<int, 16>{});
      return run(std::integral_constant<int, 32>{});
    }
    return with_experts(E, [&](auto v) {
      return with_flags([&](auto with_bias, auto with_groups) {
        return launch_overlapped(route_kernel<Type, decltype(v)::value, decltype(with_bias)::value, decltype(with_groups)::value>, dim3(route_blocks(T, kRouteBlocks<decltype(v)::value>)),
                                 dim3(32 * kRouteWarps), decltype(with_groups)::value ? (size_t)(kRouteWarps * groups * p.group_stride * 4) : 0, static_cast<cudaStream_t>(stream), 1, p);
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
  const int64_t width = E * elem_bytes(t);
  SP24_RETURN_IF(logits != dlogits && overlap({dlogits, T, width, ldd * elem_bytes(t)}, {logits, T, width, ld * elem_bytes(t)}), SP24_ERR_UNSUPPORTED);
  const sp24_status arch = check_arch();
  SP24_RETURN_IF(arch != SP24_OK, arch);
  RouteBackwardParams p = {};
  p.T = T; p.ld = ld; p.ldd = ldd; p.E = (int)E; p.k = k;
  p.sigmoid = score == SP24_SCORE_SIGMOID; p.renorm = renorm != 0; p.scale = scale;
  p.logits = logits; p.dlogits = dlogits; p.dweights = dweights; p.experts = experts;
  return with_float_type(t, [&](auto type) {
    using Type = typename decltype(type)::type;
    const int64_t es = sizeof(Type);
    if (whole_chunks(E, es, k) && aligned16(logits) && aligned16(dlogits) && (T == 1 || (ld * es % 16 == 0 && ldd * es % 16 == 0)) && T < int64_t(1) << 35) {
      auto run = [&](auto v) {
        return launch_overlapped(route_backward_chunks_kernel<Type, decltype(v)::value>, dim3((unsigned)((T + kChunkTokens - 1) / kChunkTokens)),
                                 dim3(32 * kChunkWarps), 0, static_cast<cudaStream_t>(stream), 1, p);
      };
      if (E <= 64) return run(std::integral_constant<int, 8>{});
      if (E <= 128) return run(std::integral_constant<int, 16>{});
      return run(std::integral_constant<int, 32>{});
    }
    return with_experts(E, [&](auto v) {
      return launch_overlapped(route_backward_kernel<Type, decltype(v)::value>, dim3(route_blocks(T, 8)), dim3(32 * kRouteWarps),
                               (size_t)(kRouteWarps * E * 4), static_cast<cudaStream_t>(stream), 1, p);
    });
  });
}
