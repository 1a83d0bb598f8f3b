// Scored, group-limited routing (gfx950): scores of the router's logits, a bias that
// counts for the selection only, groups of experts, top-k, gate weights; and the
// gradient of the weights to the logits.
//
//   s_e = sigmoid(z_e) or softmax(z)_e,  c_e = s_e + b_e
//   a group's score: the sum of its two largest c; the best groups are kept
//   ids: the k largest c of the kept groups, w_j = scale s_j (/ sum of the selected s)
//
// Which of two scores is larger decides whole numbers, so s and c that decide are held in
// 64 bits: c's of different experts come as near as fp32 rounds them a few times in a
// batch of 16384 tokens. The weights are rounded to fp32 once.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "launch.hpp"

namespace moe {

namespace {

constexpr int kTokens = 4;  // tokens of a block, a wave each

__device__ __forceinline__ double shfl_xor_f64(double v, int m) {
  const uint64_t u = __double_as_longlong(v);
  const uint32_t lo = __shfl_xor((uint32_t)u, m, kWave), hi = __shfl_xor((uint32_t)(u >> 32), m, kWave);
  return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}
__device__ __forceinline__ double shfl_f64(double v, int l) {
  const uint64_t u = __double_as_longlong(v);
  const uint32_t lo = __shfl((uint32_t)u, l, kWave), hi = __shfl((uint32_t)(u >> 32), l, kWave);
  return __longlong_as_double((long long)(((uint64_t)hi << 32) | lo));
}

// The score of a logit z over the factor e^m (softmax) or e^min(m, 0) (sigmoid), m the
// largest of the selected logits: what a ratio of scores needs, in range for any z.
template <bool SOFT, class F>
__device__ __forceinline__ F relative_score(float z, float m) {
  if (SOFT) return exp((F)z - (F)m);
  if (z > 0.0f) return (F)1 / ((F)1 + exp(-(F)z));
  return exp((F)z - (F)fminf(m, 0.0f)) / ((F)1 + exp((F)z));
}

// The best (value, index) of a wave: the largest value, the lowest index of equal ones.
__device__ __forceinline__ void wave_best(double& v, int& i) {
#pragma unroll
  for (int m = 1; m < kWave; m <<= 1) {
    const double ov = shfl_xor_f64(v, m);
    const int oi = __shfl_xor(i, m, kWave);
    if (ov > v || (ov == v && oi < i)) v = ov, i = oi;
  }
}

// ---------------------------------------------------------------------------
// A wave a token, lane l the experts l + 64 v. Selection by rounds of a (value, index)
// arg-max over the wave.
// ---------------------------------------------------------------------------
template <int V, bool SOFT>
__global__ __launch_bounds__(kTokens* kWave) void route_kernel(const float* __restrict__ z,
                                                               const float* __restrict__ bias,
                                                               const uint8_t* __restrict__ mask, int T, int E, int k,
                                                               int groups, int kept, int norm, double scale,
                                                               int32_t* __restrict__ ids, float* __restrict__ w) {
  __shared__ double keys[kTokens][kMaxExperts];
  __shared__ double gscore[kTokens][kMaxExperts];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long t = (long long)blockIdx.x * kTokens + wave;
  const size_t row = (size_t)(t < T ? t : T - 1);  // waves past the last token repeat it and store nothing
  const double ninf = -INFINITY;
  float zf[V];
  double s[V], key[V];
  bool bad = false;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int e = lane + 64 * v;
    zf[v] = e < E ? z[row * E + e] : -INFINITY;
    bad |= zf[v] != zf[v] || (SOFT && zf[v] == INFINITY);
  }
  bad = __any(bad);
  if (SOFT) {
    float m = -INFINITY;
#pragma unroll
    for (int v = 0; v < V; ++v) m = fmaxf(m, zf[v] == INFINITY ? -INFINITY : zf[v]);
#pragma unroll
    for (int q = 1; q < kWave; q <<= 1) m = fmaxf(m, __shfl_xor(m, q, kWave));
    double sum = 0.0;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      s[v] = zf[v] > -INFINITY && zf[v] < INFINITY ? exp((double)zf[v] - (double)m) : 0.0;
      sum += s[v];
    }
#pragma unroll
    for (int q = 1; q < kWave; q <<= 1) sum += shfl_xor_f64(sum, q);
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] = sum > 0.0 ? s[v] / sum : 0.0;
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) s[v] = 1.0 / (1.0 + exp(-(double)zf[v]));
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int e = lane + 64 * v;
    const double c = s[v] + (bias != nullptr && e < E ? (double)bias[e] : 0.0);
    const bool can = e < E && zf[v] > -INFINITY && !(SOFT && zf[v] == INFINITY) && c > ninf;  // false for a NaN
    key[v] = can ? c : ninf;
    if (e < E) keys[wave][e] = key[v];
  }
  if (groups > 1) {
    const int n = E / groups;
    __syncthreads();
    for (int g = lane; g < groups; g += kWave) {
      double a = ninf, b = ninf;  // the two largest
      for (int i = 0; i < n; ++i) {
        const double c = keys[wave][g * n + i];
        b = fmax(b, fmin(a, c));
        a = fmax(a, c);
      }
      gscore[wave][g] = b > ninf ? a + b : a;
    }
    __syncthreads();
    double gs[V];
#pragma unroll
    for (int v = 0; v < V; ++v) gs[v] = lane + 64 * v < groups ? gscore[wave][lane + 64 * v] : ninf;
    bool on[V] = {};
    for (int r = 0; r < kept; ++r) {
      double bv = ninf;
      int bi = INT32_MAX;
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (gs[v] > bv) bv = gs[v], bi = lane + 64 * v;
      wave_best(bv, bi);
      if (bv == ninf) break;  // no group with a selectable expert is left
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (lane + 64 * v == bi) gs[v] = ninf;
        on[v] |= (lane + 64 * v) / n == bi;
      }
    }
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (!on[v]) key[v] = ninf;
  }
  const bool live = mask == nullptr || mask[row] != 0;
  int my_id = -1;
  double my_s = 0.0;
  float my_z = -INFINITY;
  for (int j = 0; j < k && live; ++j) {
    double bv = ninf, bs = 0.0;
    float bz = 0.0f;
    int bi = INT32_MAX;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (key[v] > bv) bv = key[v], bi = lane + 64 * v;
    wave_best(bv, bi);
    if (bv == ninf) break;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (lane + 64 * v == bi) key[v] = ninf, bs = s[v], bz = zf[v];
    bs = shfl_f64(bs, bi & 63);
    bz = __shfl(bz, bi & 63, kWave);
    if (lane == j) my_id = bi, my_s = bs, my_z = bz;
  }
  double x = my_s;
  if (norm) {
    // the selected scores over their common factor e^m, so that ratios of scores too
    // small for 64 bits are kept
    float m = my_z;
#pragma unroll
    for (int q = 1; q < kMaxTopk; q <<= 1) m = fmaxf(m, __shfl_xor(m, q, kWave));
    x = my_id < 0 ? 0.0 : relative_score<SOFT, double>(my_z, m);
    double sum = x;
#pragma unroll
    for (int q = 1; q < kMaxTopk; q <<= 1) sum += shfl_xor_f64(sum, q);
    x = my_id < 0 ? 0.0 : x / sum;
  }
  if (lane < k && t < T) {
    x *= scale;
    if (bad && live) x = NAN;
    ids[row * k + lane] = my_id;
    w[row * k + lane] = (float)x;
  }
}

// ---------------------------------------------------------------------------
// Gradient to the logits. A wave a token: lane j < k holds slot j, lane l the
// columns l + 64 v. With d_j the gradient of slot j's weight and r_j = s_j / sum of the
// selected scores:
//   sigmoid:           dz_e = sum over slots of e of  scale d_j s_j (1 - s_j)
//   sigmoid, normed:   ... scale r_j (d_j - sum_i r_i d_i) (1 - s_j)
//   softmax, normed:   ... scale r_j (d_j - sum_i r_i d_i)   (the softmax's own sum cancels)
//   softmax:           dz_e = s_e (scale sum over slots of e of d_j - scale sum_i s_i d_i)
// Only the last reads logits that were not selected.
// ---------------------------------------------------------------------------
template <int V, bool SOFT, bool NORM>
__global__ __launch_bounds__(kTokens* kWave) void route_backward_kernel(const float* __restrict__ z,
                                                                        const int32_t* __restrict__ ids,
                                                                        const float* __restrict__ dw, int T, int E,
                                                                        int k, float scale, int accumulate,
                                                                        float* __restrict__ dz) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long t = (long long)blockIdx.x * kTokens + wave;
  if (t >= T) return;
  const size_t row = (size_t)t;
  auto sum_slots = [&](float x) {
#pragma unroll
    for (int m = 1; m < kMaxTopk; m <<= 1) x += __shfl_xor(x, m, kWave);
    return __shfl(x, 0, kWave);
  };
  int id = lane < k ? ids[row * k + lane] : -1;
  const float d = lane < k ? dw[row * k + lane] : 0.0f;
  const bool slot = id >= 0 && id < E;
  if (!slot) id = -1;
  const float zs = slot ? z[row * E + id] : -INFINITY;
  float p[V] = {};
  float val;  // what slot j adds to its expert's column
  float common = 0.0f;
  if (SOFT && !NORM) {
    float m = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) {
      const int e = lane + 64 * v;
      p[v] = e < E ? z[row * E + e] : -INFINITY;
      m = fmaxf(m, p[v]);
    }
#pragma unroll
    for (int q = 1; q < kWave; q <<= 1) m = fmaxf(m, __shfl_xor(m, q, kWave));
#pragma unroll
    for (int v = 0; v < V; ++v) {
      p[v] = m > -INFINITY ? expf(p[v] - m) : 0.0f;
      sum += p[v];
    }
#pragma unroll
    for (int q = 1; q < kWave; q <<= 1) sum += __shfl_xor(sum, q, kWave);
    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) p[v] *= inv;
    const float ps = slot && m > -INFINITY ? expf(zs - m) * inv : 0.0f;
    val = slot ? scale * d : 0.0f;
    common = sum_slots(slot ? val * ps : 0.0f);
  } else {
    float r, x = slot ? d : 0.0f;
    if (NORM) {
      float m = zs;
#pragma unroll
      for (int q = 1; q < kMaxTopk; q <<= 1) m = fmaxf(m, __shfl_xor(m, q, kWave));
      r = slot && m > -INFINITY ? relative_score<SOFT, float>(zs, m) : 0.0f;
      const float sum = sum_slots(r);
      r = sum != 0.0f ? r / sum : 0.0f;  // no slot has an expert, or they are -inf
      x -= sum_slots(slot ? r * x : 0.0f);
    } else {
      r = slot ? 1.0f / (1.0f + expf(-zs)) : 0.0f;
    }
    const float rest = SOFT ? 1.0f : 1.0f / (1.0f + expf(zs));
    val = slot ? scale * r * x * rest : 0.0f;
  }
  float out[V] = {};
  for (int j = 0; j < k; ++j) {
    const int e = __shfl(id, j, kWave);
    const float a = __shfl(val, j, kWave);
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (lane + 64 * v == e) out[v] += a;
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int e = lane + 64 * v;
    if (e < E) {
      float x = SOFT && !NORM ? p[v] * (out[v] - common) : out[v];
      if (accumulate) x += dz[row * E + e];
      dz[row * E + e] = x;
    }
  }
}

}  // namespace

// Tokens of a launch: its threads stay below 2^32.
constexpr int kLaunchTokens = 1 << 24;

hipError_t launch_route(const float* z, const float* bias, const uint8_t* mask, int T, int E, int k, bool softmax,
                        int groups, int kept, bool norm, double scale, int32_t* ids, float* w, hipStream_t s) {
  if (kept >= groups) groups = kept = 1;  // every group is kept
  for (int t0 = 0; t0 < T;) {
    const int n = std::min(T - t0, kLaunchTokens);
    const dim3 grid((unsigned)((n - 1) / kTokens + 1)), block(kTokens * kWave);
    auto go = [&](auto kernel) {
      kernel<<<grid, block, 0, s>>>(z + (size_t)t0 * E, bias, mask ? mask + t0 : nullptr, n, E, k, groups, kept,
                                    norm ? 1 : 0, scale, ids + (size_t)t0 * k, w + (size_t)t0 * k);
    };
    switch ((E - 1) / kWave) {
      case 0: softmax ? go(route_kernel<1, true>) : go(route_kernel<1, false>); break;
      case 1: softmax ? go(route_kernel<2, true>) : go(route_kernel<2, false>); break;
      case 2: softmax ? go(route_kernel<3, true>) : go(route_kernel<3, false>); break;
      default: softmax ? go(route_kernel<4, true>) : go(route_kernel<4, false>); break;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    t0 += n;
  }
  return hipSuccess;
}

hipError_t launch_route_backward(const float* z, const int32_t* ids, const float* dw, int T, int E, int k,
                                 bool softmax, bool norm, float scale, bool accumulate, float* dz, hipStream_t s) {
  for (int t0 = 0; t0 < T;) {
    const int n = std::min(T - t0, kLaunchTokens);
    const dim3 grid((unsigned)((n - 1) / kTokens + 1)), block(kTokens * kWave);
    auto go = [&](auto kernel) {
      kernel<<<grid, block, 0, s>>>(z + (size_t)t0 * E, ids + (size_t)t0 * k, dw + (size_t)t0 * k, n, E, k, scale,
                                    accumulate ? 1 : 0, dz + (size_t)t0 * E);
    };
    auto kind = [&](auto vv) {
      constexpr int V = decltype(vv)::value;
      if (softmax)
        norm ? go(route_backward_kernel<V, true, true>) : go(route_backward_kernel<V, true, false>);
      else
        norm ? go(route_backward_kernel<V, false, true>) : go(route_backward_kernel<V, false, false>);
    };
    switch ((E - 1) / kWave) {
      case 0: kind(std::integral_constant<int, 1>{}); break;
      case 1: kind(std::integral_constant<int, 2>{}); break;
      case 2: kind(std::integral_constant<int, 3>{}); break;
      default: kind(std::integral_constant<int, 4>{}); break;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    t0 += n;
  }
  return hipSuccess;
}

}  // namespace moe
