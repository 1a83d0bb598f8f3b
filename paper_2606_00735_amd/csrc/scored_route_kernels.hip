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
// batch of 16384 tokens. The weights of what is selected are computed in 64 bits as well and
// rounded to fp32 once.
#include <math.h>

#include <algorithm>
#include <type_traits>
#include <utility>

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
  const F over = exp((F)z - (F)fminf(m, 0.0f)), e = exp(z > 0.0f ? -(F)z : (F)z);  // without a branch: side by side
  return (z > 0.0f ? (F)1 : over) / ((F)1 + e);
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
// Sixteen lanes a token, lane l the experts l V .. l V + V - 1: any number of experts without
// groups, and groups of one, two, four, eight or sixteen whole lanes of 1, 2, 4, 8, 10, 12 or 16
// experts (lane_experts).
//
// The selection runs on 32-bit keys: c in fp32 (an exponential and a reciprocal of 1 ulp),
// mapped to integers in the same order, the lowest 4 bits replaced by the position in the
// lane. A lane sorts its keys once; a round is then a maximum of the lanes' first ones (four
// DPP steps), and the lane that had it takes its next one. k rounds run without a look at
// their gaps, which the lanes see to afterwards, a candidate each.
//
// What fp32 cannot decide is seen from the gaps (`wide`: more than twice what a key can be
// off). Rounds go on until the next key is certainly below the k-th best, so that the k
// best are among the candidates; where a gap between candidates is not wide, their c's are
// computed in 64 bits, two a lane, and ordered by rank. So are the groups' scores where the
// border of the kept ones is not certain. Only a token with more than 32 candidates, three
// c's of a lane alike at that border, a NaN or an infinite score selects again from all its
// experts in 64 bits.
// 16384 tokens x 256 experts, 4 of 8 groups: 61 us with every row in 64 bits, a wave each;
// 37 us without the sort and with all uncertain rows done again; 13.6 us with the gaps in the
// rounds and the keys moved through registers; 11.4-11.8 us so, the logits in the last-level
// cache (from memory 13.0; one token 4.7). A wave of four tokens has 960 vector instructions, four
// waves a SIMD run at once: 15 400 cycles of issue of the 25 900 that a CU is busy.
// ---------------------------------------------------------------------------
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t x) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
}
template <int CTRL>
__device__ __forceinline__ float dpp_f(float x) {
  return __uint_as_float(dpp_u32<CTRL>(__float_as_uint(x)));
}
// over 16 lanes; every lane gets the result
template <class T, class Op>
__device__ __forceinline__ T row_reduce(T x, Op op) {
  auto at = [&](auto step) {
    constexpr int C = decltype(step)::value;
    if constexpr (std::is_same<T, float>::value)
      return dpp_f<C>(x);
    else
      return dpp_u32<C>(x);
  };
  x = op(x, at(std::integral_constant<int, 0xB1>{}));   // quad_perm 1,0,3,2
  x = op(x, at(std::integral_constant<int, 0x4E>{}));   // quad_perm 2,3,0,1
  x = op(x, at(std::integral_constant<int, 0x141>{}));  // row_half_mirror
  x = op(x, at(std::integral_constant<int, 0x140>{}));  // row_mirror
  return x;
}
__device__ __forceinline__ float row_max(float x) {
  return row_reduce(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float row_min(float x) {
  return row_reduce(x, [](float a, float b) { return fminf(a, b); });
}
__device__ __forceinline__ float row_sum(float x) {
  return row_reduce(x, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ double row_sum64(double x) {
  auto plus = [&](auto step) {
    constexpr int C = decltype(step)::value;
    const uint64_t u = (uint64_t)__double_as_longlong(x);
    const uint64_t o = (uint64_t)dpp_u32<C>((uint32_t)u) | ((uint64_t)dpp_u32<C>((uint32_t)(u >> 32)) << 32);
    x += __longlong_as_double((long long)o);
  };
  plus(std::integral_constant<int, 0xB1>{});   // as row_reduce
  plus(std::integral_constant<int, 0x4E>{});
  plus(std::integral_constant<int, 0x141>{});
  plus(std::integral_constant<int, 0x140>{});
  return x;
}

// f(std::integral_constant<int, q>) for every q of the sequence
template <class F, int... Q>
__device__ __forceinline__ void for_each_int(F&& f, std::integer_sequence<int, Q...>) {
  (f(std::integral_constant<int, Q>{}), ...);
}

// fp32 in the order of unsigned integers; 0 is below every number
__device__ __forceinline__ uint32_t order_key(float c) {
  const uint32_t u = __float_as_uint(c);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
  const uint32_t u = k & ~15u;
  return __uint_as_float((u & 0x80000000u) ? u ^ 0x80000000u : ~u);
}

__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }

struct RouteArgs {
  const float* z;
  const float* bias;
  const uint8_t* mask;
  int T, E, k;
  int groups, kept;  // groups 1: no grouping
  int norm;
  double scale;
  int32_t* ids;
  float* w;
};

// Sorts V keys of a lane, the largest first (odd-even merges, the size rounded up to a
// power of two with zeros that the compiler drops).
template <int V>
__device__ __forceinline__ void sort_keys(uint32_t (&key)[V]) {
  constexpr int P = V <= 1 ? 1 : V <= 2 ? 2 : V <= 4 ? 4 : V <= 8 ? 8 : 16;
  uint32_t x[P];
#pragma unroll
  for (int v = 0; v < P; ++v) x[v] = v < V ? key[v % V] : 0u;
#pragma unroll
  for (int p = 1; p < P; p *= 2)
#pragma unroll
    for (int d = p; d >= 1; d /= 2)
#pragma unroll
      for (int j = d % p; j + d < P; j += 2 * d)
#pragma unroll
        for (int i = 0; i < d; ++i)
          if (i + j + d < P && (i + j) / (2 * p) == (i + j + d) / (2 * p)) {
            const uint32_t a = x[i + j], b = x[i + j + d];
            x[i + j] = max(a, b);
            x[i + j + d] = min(a, b);
          }
#pragma unroll
  for (int v = 0; v < V; ++v) key[v] = x[v];
}

// The selection of a token in 64 bits: this lane's slot (lane l: slot l) in id and its
// logit in zsel; bad: the row has a NaN or an infinite score. All 64 lanes call it, tokens of their own every 16. Keys
// are in LDS, a lane's own at keys[256 v], and every loop is rolled: rarely run, it is to
// take neither registers nor code from what surrounds it.
template <int V, bool SOFT>
__device__ __forceinline__ void select64(const RouteArgs& a, const float* row, int l, bool live, double* keys, int& id,
                                         float& zsel, bool& bad) {
  const double ninf = -INFINITY;
  const int E = a.E;
  auto logit = [&](int v) { return l * V + v < E ? row[l * V + v] : -INFINITY; };
  float m = -INFINITY;
  bad = false;
#pragma unroll 1
  for (int v = 0; v < V; ++v) {
    const float z = logit(v);
    const bool out = z != z || (SOFT && z == INFINITY);
    bad |= out;
    if (!out) m = fmaxf(m, z);
  }
  m = row_max(m);
  bad = row_max(bad ? 1.0f : 0.0f) != 0.0f;
  auto rises = [](float z) { return z > -INFINITY && z < INFINITY; };
  double sum = 0.0;
  if (SOFT) {
#pragma unroll 1
    for (int v = 0; v < V; ++v) {
      const float z = logit(v);
      sum += rises(z) ? exp((double)z - (double)m) : 0.0;
    }
    sum = row_sum64(sum);
  }
  auto score = [&](float z) {
    if (SOFT) return rises(z) ? exp((double)z - (double)m) / sum : 0.0;
    return 1.0 / (1.0 + exp(-(double)z));
  };
  double x = ninf, y = ninf;  // the two largest of the lane, then of the group
#pragma unroll 1
  for (int v = 0; v < V; ++v) {
    const int e = l * V + v;
    const float z = logit(v);
    const double c = score(z) + (a.bias != nullptr && e < E ? (double)a.bias[e] : 0.0);
    const double key = z > -INFINITY && !(SOFT && z == INFINITY) && c > ninf ? c : ninf;
    keys[256 * v] = key;
    y = fmax(y, fmin(x, key));
    x = fmax(x, key);
  }
  bool on = true;
  if (a.groups > 1) {
    const int LG = 16 / a.groups;
#pragma unroll 1
    for (int q = 1; q < LG; q <<= 1) {
      const double ox = shfl_xor_f64(x, q), oy = shfl_xor_f64(y, q);
      y = fmax(fmin(x, ox), fmax(y, oy));
      x = fmax(x, ox);
    }
    const double mine = y > ninf ? x + y : x;
    int before = 0;  // lanes of groups that come before this one
#pragma unroll 1
    for (int q = 1; q < 16; ++q) {
      const double other = shfl_xor_f64(mine, q);
      before += other > mine || (other == mine && (l ^ q) / LG < l / LG);
    }
    on = before < a.kept * LG;
  }
  id = -1;
  zsel = -INFINITY;
#pragma unroll 1
  for (int j = 0; j < a.k; ++j) {
    double bv = ninf;
    int bi = INT32_MAX;
#pragma unroll 1
    for (int v = 0; v < V; ++v) {
      const double key = on ? keys[256 * v] : ninf;
      if (key > bv) bv = key, bi = l * V + v;
    }
#pragma unroll 1
    for (int q = 1; q < 16; q <<= 1) {
      const double ov = shfl_xor_f64(bv, q);
      const int oi = __shfl_xor(bi, q, kWave);
      if (ov > bv || (ov == bv && oi < bi)) bv = ov, bi = oi;
    }
    if (bv > ninf) {
      if (bi / V == l) keys[256 * (bi % V)] = ninf;
      if (l == j && live) id = bi, zsel = row[bi];
    }
  }
}

template <int V, bool SOFT>
__global__ __launch_bounds__(256) void route_rows_kernel(RouteArgs a) {
  __shared__ double keys64[V * 256];  // of select64, and sorted 32-bit keys
  const int lane = threadIdx.x & 63, l = lane & 15;
  const long long t = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
  const size_t r = (size_t)(t < a.T ? t : a.T - 1);  // lanes past the last token repeat it and store nothing
  const int E = a.E, e0 = l * V;
  const float* row = a.z + r * (size_t)E;
  float z[V];
  if (V % 4 == 0 && E % 4 == 0) {
#pragma unroll
    for (int v = 0; v < V / 4; ++v) {
      float4 q = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
      if (e0 + 4 * v < E) q = *reinterpret_cast<const float4*>(row + e0 + 4 * v);
      z[4 * v % V] = q.x, z[(4 * v + 1) % V] = q.y, z[(4 * v + 2) % V] = q.z, z[(4 * v + 3) % V] = q.w;
    }
  } else {
#pragma unroll
    for (int v = 0; v < V; ++v) z[v] = e0 + v < E ? row[e0 + v] : -INFINITY;
  }
  const bool live = a.mask == nullptr || a.mask[r] != 0;
  const bool biased = a.bias != nullptr;
  float bias[V];
  if (biased) {
    if (V % 4 == 0 && E % 4 == 0 && (reinterpret_cast<uintptr_t>(a.bias) & 15u) == 0) {
#pragma unroll
      for (int v = 0; v < V / 4; ++v) {
        float4 q = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (e0 + 4 * v < E) q = *reinterpret_cast<const float4*>(a.bias + e0 + 4 * v);
        bias[4 * v % V] = q.x, bias[(4 * v + 1) % V] = q.y, bias[(4 * v + 2) % V] = q.z, bias[(4 * v + 3) % V] = q.w;
      }
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) bias[v] = e0 + v < E ? a.bias[e0 + v] : 0.0f;
    }
  }
  // range of the row's finite logits; ok: no NaN, no +inf
  float hi = -INFINITY, lo = INFINITY;
  bool ok = true;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    ok &= z[v] < INFINITY;
    hi = fmaxf(hi, z[v]);
    lo = fminf(lo, z[v] > -INFINITY ? z[v] : INFINITY);
  }
  hi = row_max(hi), lo = row_min(lo);
  ok = ((uint32_t)(__ballot(ok) >> (lane & 48)) & 0xffffu) == 0xffffu;  // of the row, as all that is and-ed to it below
  // What a score can be off, relative to it. sigmoid: the argument of the exponential (its
  // product with log2 e, 1.5 2^-24 of it), 1 ulp each of exponential and reciprocal, a sum.
  // softmax: a difference in the argument, too, and a sum of up to 20 steps.
  const float span = fminf(SOFT ? hi - lo : fmaxf(fabsf(hi), fabsf(lo)), 128.0f);
  const float rel = SOFT ? 0x1p-19f + span * 0x1p-22f : 0x1p-21f + span * 0x1p-23f;
  uint32_t key[V];
  float inv = 1.0f, top = 1.0f;  // 1 / sum, the largest score
  if (SOFT) {
    float sum = 0.0f;
#pragma unroll
    for (int v = 0; v < V; ++v) sum += z[v] > -INFINITY ? exp_fast(z[v] - hi) : 0.0f;
    sum = row_sum(sum);
    inv = __builtin_amdgcn_rcpf(sum);
    top = inv;
  }
  // The softmax's sum in 64 bits (over e^hi): weights that are not normed need it, c's beside a
  // bias where they decide.
  double total = 1.0;
  bool have_total = false;
  if (SOFT && !a.norm) {
    have_total = true;
    total = 0.0;
#pragma unroll
    for (int v = 0; v < V; ++v) total += exp(fmax((double)z[v] - (double)hi, -800.0));  // 0 of -inf, without a branch
    total = row_sum64(total);
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float c = SOFT ? exp_fast(z[v] - hi) * inv : __builtin_amdgcn_rcpf(1.0f + exp_fast(-z[v]));
    if (biased) c += bias[v];
    key[v] = z[v] > -INFINITY && c > -INFINITY ? (order_key(c) & ~15u) | (uint32_t)(15 - v) : 0u;
  }
  // twice what two keys' values, at most x and at most y in size, can differ by from
  // their exact ones: the 4 bits, the sum with the bias, the scores
  auto wide = [&](float gap, float x, float y) {
    const float size = fmaxf(fabsf(x), fabsf(y));
    return gap > 2.0f * (size * 0x1.1p-19f + rel * (biased ? top : size)) + 0x1p-120f;
  };
  sort_keys<V>(key);
  // c of an expert in 64 bits. A softmax's sum counts beside a bias only.
  auto exact = [&](int e) {
    const double zd = (double)row[e];
    const double sc = SOFT ? exp(zd - (double)hi) / total : 1.0 / (1.0 + exp(-zd));
    return biased ? sc + (double)a.bias[e] : sc;
  };
  auto sum_scores = [&] {
    if (!SOFT || have_total) return;
    have_total = true;
    total = 0.0;
#pragma unroll 1
    for (int v = 0; v < V; ++v) {
      const float zv = e0 + v < E ? row[e0 + v] : -INFINITY;
      total += zv > -INFINITY ? exp((double)zv - (double)hi) : 0.0;
    }
    total = row_sum64(total);
  };
  auto expert_of = [&](uint32_t k) { return e0 + 15 - (int)(k & 15u); };
  if (a.groups > 1) {
    uint32_t x = key[0], y = V > 1 ? key[1 % V] : 0u;  // the two largest of the group
    const int LG = 16 / a.groups;
    auto join = [&](uint32_t ox, uint32_t oy) {
      y = max(min(x, ox), max(y, oy));
      x = max(x, ox);
    };
    if (LG >= 2) join(dpp_u32<0xB1>(x), dpp_u32<0xB1>(y));
    if (LG >= 4) join(dpp_u32<0x4E>(x), dpp_u32<0x4E>(y));
    if (LG >= 8) join(dpp_u32<0x141>(x), dpp_u32<0x141>(y));
    const float vx = x ? key_value(x) : -INFINITY, vy = y ? key_value(y) : 0.0f;
    const float score = vx + vy, size = x ? fabsf(vx) + fabsf(vy) : 0.0f;
    int before = 0;  // lanes of groups with a larger score
    auto see = [&](float os) { before += os > score; };
    see(dpp_f<0x121>(score)), see(dpp_f<0x122>(score)), see(dpp_f<0x123>(score)), see(dpp_f<0x124>(score));
    see(dpp_f<0x125>(score)), see(dpp_f<0x126>(score)), see(dpp_f<0x127>(score)), see(dpp_f<0x128>(score));
    see(dpp_f<0x129>(score)), see(dpp_f<0x12A>(score)), see(dpp_f<0x12B>(score)), see(dpp_f<0x12C>(score));
    see(dpp_f<0x12D>(score)), see(dpp_f<0x12E>(score)), see(dpp_f<0x12F>(score));
    // a group with nothing to select is not kept
    bool on = x != 0 && before < a.kept * LG;
    const int many = __popc((uint32_t)(__ballot(on) >> (lane & 48)) & 0xffffu);
    const float in = row_min(on ? score : INFINITY), out = row_max(on ? -INFINITY : score);
    const float all = row_max(size);
    // Each score has the errors of two values (their sum's rounding is within the 0x1.1).
    // More lanes than those of the groups to keep: equal scores at the border.
    const bool sure = many <= a.kept * LG && (out == -INFINITY || wide((in - out) * 0.5f, all, all));
    if (__any(live && !sure)) {
      // the scores in 64 bits, of a lane's two largest c's: they are among its three
      // largest keys where the fourth is certainly below the second
      if (biased || SOFT) sum_scores();
      const double ninf = -INFINITY;
      double p = ninf, q = ninf;
#pragma unroll
      for (int v = 0; v < (V < 3 ? V : 3); ++v) {
        const double c = key[v] ? exact(expert_of(key[v])) : ninf;
        q = fmax(q, fmin(p, c));
        p = fmax(p, c);
      }
      if (V > 3) {
        const float second = key_value(key[1 % V]), fourth = key_value(key[3 % V]);
        const bool clear = key[3 % V] == 0 || wide(second - fourth, second, fourth);
        const bool clears = row_max(clear ? 0.0f : 1.0f) == 0.0f;
        ok &= sure || clears;
      }
#pragma unroll 1
      for (int d = 1; d < LG; d <<= 1) {
        const double op = shfl_xor_f64(p, d), oq = shfl_xor_f64(q, d);
        q = fmax(fmin(p, op), fmax(q, oq));
        p = fmax(p, op);
      }
      const double mine = q > ninf ? p + q : p;
      int first = 0;  // lanes of groups that come before this one
#pragma unroll
      for (int d = 1; d < 16; ++d) {
        const double other = shfl_xor_f64(mine, d);
        first += other > mine || (other == mine && (l ^ d) / LG < l / LG);
      }
      if (!sure) on = x != 0 && first < a.kept * LG;
    }
    if (!on) {
#pragma unroll
      for (int v = 0; v < V; ++v) key[v] = 0;
    }
  }
  // The largest key of the row, k times and then as long as one may belong before the k-th.
  // A lane's two largest left are in registers, the others in LDS (sixteen registers moved up
  // were a third of a round).
  constexpr bool kInLds = V > 4;
  uint32_t k0 = key[0], k1 = V > 1 ? key[1 % V] : 0u;
  // in the thread's own doubles: another wave may be in select64
  typedef uint32_t __attribute__((may_alias)) word;
  word* rest = reinterpret_cast<word*>(keys64 + threadIdx.x);
  if (kInLds) {
#pragma unroll
    for (int v = 0; v < V; ++v) rest[512 * v] = v + 2 < V ? key[(v + 2) % V] : 0u;
  }
  // takes the largest, which is not 0: its expert; of equal keys of several lanes, the
  // lowest lane's
  auto take = [&](uint32_t best) __attribute__((always_inline)) {
    const int holder = __ffs((uint32_t)(__ballot(k0 == best) >> (lane & 48)) & 0xffffu) - 1;
    if (l == holder && best != 0) {
      k0 = k1;
      if (kInLds) {
        k1 = *rest;
        rest += 512;
      } else {
#pragma unroll
        for (int v = 1; v + 1 < V; ++v) key[v] = key[v + 1];
        key[V - 1] = 0;
        k1 = V > 1 ? key[1 % V] : 0u;
      }
    }
    return holder * V + 15 - (int)(best & 15u);
  };
  auto largest = [&] { return row_reduce(k0, [](uint32_t p, uint32_t q) { return max(p, q); }); };
  int id = -1, id2 = -1;  // candidates l and 16 + l
  uint32_t mine = 0, best = 0;  // candidate l's key, the last one's
#pragma unroll 1
  for (int j = 0; j < a.k; ++j) {
    best = largest();
    const int e = take(best);
    if (l == j && best != 0) id = e, mine = best;
  }
  // near: a gap between candidates is not wide
  const float value = key_value(mine), prev = key_value(dpp_u32<0x111>(mine));  // row_shr by 1
  bool near = l > 0 && mine != 0 && !wide(prev - value, prev, value);
  if (best != 0) {
    const float kth = key_value(best);
#pragma unroll 1
    for (int j = a.k;; ++j) {
      best = largest();
      const float v = key_value(best);
      if (best == 0 || wide(kth - v, kth, v)) break;
      if (j == 32) {
        ok = false;
        break;
      }
      near = true;
      const int e = take(best);
      if (l == j) id = e;
      if (l + 16 == j) id2 = e;
    }
  }
  if (__any(live && near && ok)) {
    if (biased) sum_scores();
    const double c = id >= 0 ? exact(id) : -INFINITY;
    if (!__any(id2 >= 0)) {
      int rank = 0;
      auto see = [&](auto step) {
        constexpr int C = 0x121 + decltype(step)::value;  // row_ror by 1 to 15
        const uint64_t u = (uint64_t)__double_as_longlong(c);
        const uint64_t o = (uint64_t)dpp_u32<C>((uint32_t)u) | ((uint64_t)dpp_u32<C>((uint32_t)(u >> 32)) << 32);
        const double oc = __longlong_as_double((long long)o);
        const int oid = (int)dpp_u32<C>((uint32_t)id);
        rank += oc > c || (oc == c && oid < id);
      };
      for_each_int(see, std::make_integer_sequence<int, 15>{});
      if (id < 0) rank = l;  // lanes without a candidate stay behind the others
      id = __builtin_amdgcn_ds_permute(((lane & 48) + rank) * 4, id);
    } else {
      const double c2 = id2 >= 0 ? exact(id2) : -INFINITY;
      int rank = 0, rank2 = 0;
#pragma unroll 1
      for (int q = 0; q < 16; ++q) {
        const double oc = shfl_xor_f64(c, q), oc2 = shfl_xor_f64(c2, q);
        const int oid = __shfl_xor(id, q, kWave), oid2 = __shfl_xor(id2, q, kWave);
        rank += (oc > c || (oc == c && oid < id)) + (oc2 > c || (oc2 == c && oid2 < id));
        rank2 += (oc > c2 || (oc == c2 && oid < id2)) + (oc2 > c2 || (oc2 == c2 && oid2 < id2));
      }
      int put = -1;  // the lane of a place looks for its candidate
#pragma unroll 1
      for (int q = 0; q < 16; ++q) {
        const int orank = __shfl_xor(rank, q, kWave), orank2 = __shfl_xor(rank2, q, kWave);
        const int oid = __shfl_xor(id, q, kWave), oid2 = __shfl_xor(id2, q, kWave);
        if (oid >= 0 && orank == l) put = oid;
        if (oid2 >= 0 && orank2 == l) put = oid2;
      }
      id = put;
    }
  }
  if (l >= a.k) id = -1;
  float zs = id >= 0 ? row[id] : -INFINITY;
  bool bad = false;
  if (__any(live && !ok)) {
    int id64;
    float zs64;
    select64<V, SOFT>(a, row, l, live, keys64 + threadIdx.x, id64, zs64, bad);
    if (!ok) id = id64, zs = zs64;
  }
  if (!live) id = -1;
  // Weights in 64 bits, by one formula whatever path has selected, rounded once (in fp32 they
  // were off by one or two roundings more; it costs 0.2 us of 16384 x 256, and 3.0 where the softmax's
  // sum has to be in 64 bits, too: 7.9 -> 10.9 without groups, as many exponentials as scores; 12.9
  // with a branch around each).
  const bool slot = l < a.k && id >= 0;
  double x, sum = 1.0;
  if (a.norm) {
    const float m = row_max(slot ? zs : -INFINITY);
    x = slot ? relative_score<SOFT, double>(zs, m) : 0.0;
    sum = row_sum64(x);
  } else if (SOFT) {
    x = exp((double)zs - (double)hi);
    sum = total;
  } else {
    x = 1.0 / (1.0 + exp(-(double)zs));
  }
  x = slot ? x / sum * a.scale : 0.0;
  if (bad && live) x = NAN;
  if (l < a.k && t < a.T) {
    a.ids[r * a.k + l] = id;
    a.w[r * a.k + l] = (float)x;
  }
}

// ---------------------------------------------------------------------------
// Gradient to the logits. Sixteen lanes a token: lane j < k holds slot j, lane l the
// columns 64 q + 4 l .. + 3. With d_j the gradient of slot j's weight and r_j = s_j / sum of
// the selected scores:
//   sigmoid:           dz_e = sum over slots of e of  scale d_j s_j (1 - s_j)
//   sigmoid, normed:   ... scale r_j (d_j - sum_i r_i d_i) (1 - s_j)
//   softmax, normed:   ... scale r_j (d_j - sum_i r_i d_i)   (the softmax's own sum cancels)
//   softmax:           dz_e = s_e (scale sum over slots of e of d_j - scale sum_i s_i d_i)
// Only the last reads logits that were not selected. The slots' values reach their columns
// through a row of zeros in LDS (slots of the same expert are added up first, in their
// order), which leaves as whole lines. The row of zeros is what it costs: 16384 x 256, 17
// MB, a wave a token with a comparison of every slot with every column 9.8 us.
// ---------------------------------------------------------------------------
template <int Q, bool SOFT, bool NORM>
__global__ __launch_bounds__(256) void route_backward_kernel(const float* __restrict__ z,
                                                             const int32_t* __restrict__ ids,
                                                             const float* __restrict__ dw, int T, int E, int k,
                                                             float scale, int accumulate, float* __restrict__ dz) {
  __shared__ __align__(16) float rows[16][64 * Q];
  const int l = threadIdx.x & 15, tok = threadIdx.x >> 4;
  const long long t = (long long)blockIdx.x * 16 + tok;
  const bool in = t < T;
  const size_t row = (size_t)(in ? t : T - 1);  // lanes past the last token repeat it and store nothing
  const bool vec = E % 4 == 0;
  float4* mine = reinterpret_cast<float4*>(rows[tok]);
#pragma unroll
  for (int q = 0; q < Q; ++q) mine[16 * q + l] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  int id = l < k ? ids[row * k + l] : -1;
  const float d = l < k ? dw[row * k + l] : 0.0f;
  const bool slot = id >= 0 && id < E;
  if (!slot) id = -1;
  const float zs = slot ? z[row * E + id] : -INFINITY;
  float p[Q][4] = {};
  float val, common = 0.0f;  // what slot l adds to its expert's column
  // A token without any expert has no gradient, whatever its logits hold (a softmax's NaN
  // would pass through a product with 0).
  const bool none = SOFT && !NORM && row_max(slot ? 1.0f : 0.0f) == 0.0f;
  if (SOFT && !NORM) {
    float m = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const int e = 64 * q + 4 * l;
      float4 v = make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
      const float* pz = z + row * E + e;
      if (vec) {
        if (e < E) v = *reinterpret_cast<const float4*>(pz);
      } else {
        if (e < E) v.x = pz[0];
        if (e + 1 < E) v.y = pz[1];
        if (e + 2 < E) v.z = pz[2];
        if (e + 3 < E) v.w = pz[3];
      }
      p[q][0] = v.x, p[q][1] = v.y, p[q][2] = v.z, p[q][3] = v.w;
      m = fmaxf(m, fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)));
    }
    m = row_max(m);
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        p[q][c] = m > -INFINITY ? expf(p[q][c] - m) : 0.0f;
        sum += p[q][c];
      }
    sum = row_sum(sum);
    const float inv = sum > 0.0f || sum != sum ? 1.0f / sum : 0.0f;
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int c = 0; c < 4; ++c) p[q][c] *= inv;
    const float ps = slot && m > -INFINITY ? expf(zs - m) * inv : 0.0f;
    val = slot ? scale * d : 0.0f;
    common = row_sum(slot ? val * ps : 0.0f);
  } else {
    float r, x = slot ? d : 0.0f;
    if (NORM) {
      const float m = row_max(zs);
      r = slot && m > -INFINITY ? relative_score<SOFT, float>(zs, m) : 0.0f;
      const float sum = row_sum(r);
      r = sum != 0.0f ? r / sum : 0.0f;  // no slot has an expert, or they are -inf
      x -= row_sum(slot ? r * x : 0.0f);
    } else {
      r = slot ? relative_score<false, float>(zs, 0.0f) : 0.0f;
    }
    const float rest = SOFT ? 1.0f : 1.0f / (1.0f + expf(zs));
    val = slot ? scale * r * x * rest : 0.0f;
  }
  // slots of one expert: the first of them has their sum, in their order
  float total = 0.0f;
  bool first = slot;
  for_each_int(
      [&](auto j) {
        constexpr int J = decltype(j)::value;
        const int oid = (int)dpp_u32<0x150 + J>((uint32_t)id);  // row_newbcast
        const float ov = dpp_f<0x150 + J>(val);
        if (oid == id) {
          total += ov;
          first &= J >= l;
        }
      },
      std::make_integer_sequence<int, kMaxTopk>{});
  if (first) rows[tok][id] = total;
  // a wave reads what it has written; LDS serves a wave in order
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  if (!in) return;
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int e = 64 * q + 4 * l;
    const float4 f = mine[16 * q + l];
    float v[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (SOFT && !NORM) v[c] = none ? 0.0f : p[q][c] * (v[c] - common);
    float* out = dz + row * E + e;
    if (vec) {
      if (e < E) {
        if (accumulate) {
          const float4 o = *reinterpret_cast<const float4*>(out);
          v[0] += o.x, v[1] += o.y, v[2] += o.z, v[3] += o.w;
        }
        *reinterpret_cast<float4*>(out) = make_float4(v[0], v[1], v[2], v[3]);
      }
    } else {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        if (e + c < E) out[c] = accumulate ? out[c] + v[c] : v[c];
    }
  }
}

}  // namespace

// Tokens of a launch: its threads stay below 2^32.
constexpr int kLaunchTokens = 1 << 24;

// Experts of a lane in route_rows_kernel, or 0 where it does not apply: without groups any
// count; with groups E = 16 V, and the groups whole lanes, for the V that are compiled. Other
// counts take route_kernel even where their groups would be whole lanes: 16384 tokens by 96
// experts in 8 groups (V = 6) 39.8 us, by 128 experts 8.4.
static int lane_experts(int E, int groups) {
  for (int V : {1, 2, 4, 8, 10, 12, 16})
    if (groups == 1 ? 16 * V >= E : 16 * V == E && 16 % groups == 0) return V;
  return 0;
}

hipError_t launch_route(const float* z, const float* bias, const uint8_t* mask, int T, int E, int k, bool softmax,
                        int groups, int kept, bool norm, double scale, int32_t* ids, float* w, hipStream_t s) {
  if (kept >= groups) groups = kept = 1;  // every group is kept
  for (int t0 = 0; t0 < T;) {
    const int n = std::min(T - t0, kLaunchTokens);
    const dim3 grid((unsigned)((n - 1) / kTokens + 1)), block(kTokens * kWave);
    const int V = lane_experts(E, groups);
    if (V > 0) {
      const RouteArgs a{z + (size_t)t0 * E, bias, mask ? mask + t0 : nullptr, n, E, k, groups, kept, norm ? 1 : 0, scale,
                        ids + (size_t)t0 * k, w + (size_t)t0 * k};
      const unsigned blocks = (unsigned)((n - 1) / 16 + 1);
      auto rows = [&](auto vv) {
        constexpr int W = decltype(vv)::value;
        if (softmax)
          route_rows_kernel<W, true><<<blocks, 256, 0, s>>>(a);
        else
          route_rows_kernel<W, false><<<blocks, 256, 0, s>>>(a);
      };
      switch (V) {
        case 1: rows(std::integral_constant<int, 1>{}); break;
        case 2: rows(std::integral_constant<int, 2>{}); break;
        case 4: rows(std::integral_constant<int, 4>{}); break;
        case 8: rows(std::integral_constant<int, 8>{}); break;
        case 10: rows(std::integral_constant<int, 10>{}); break;
        case 12: rows(std::integral_constant<int, 12>{}); break;
        default: rows(std::integral_constant<int, 16>{}); break;
      }
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      t0 += n;
      continue;
    }
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
    const unsigned blocks = (unsigned)((n - 1) / 16 + 1);
    auto go = [&](auto kernel) {
      kernel<<<blocks, 256, 0, s>>>(z + (size_t)t0 * E, ids + (size_t)t0 * k, dw + (size_t)t0 * k, n, E, k, scale,
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
