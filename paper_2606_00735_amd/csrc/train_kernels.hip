// The router's training step (gfx950): balance and z losses with per-expert
// counts, the gradient to the router logits, and the gradient of the weighted
// combine.
#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "launch.hpp"

namespace moe {

// ---------------------------------------------------------------------------
// Lane reductions without LDS: DPP within 16 lanes, row swaps beyond. Every lane
// of an aligned group of L ends with the result; all lanes must be active.
// ---------------------------------------------------------------------------
template <int CTRL>
__device__ __forceinline__ float dpp_f32(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <int L, class Op>
__device__ __forceinline__ float group_reduce(float x, Op op) {
  if (L >= 2) x = op(x, dpp_f32<0xB1>(x));    // quad_perm 1,0,3,2
  if (L >= 4) x = op(x, dpp_f32<0x4E>(x));    // quad_perm 2,3,0,1
  if (L >= 8) x = op(x, dpp_f32<0x141>(x));   // row_half_mirror
  if (L >= 16) x = op(x, dpp_f32<0x140>(x));  // row_mirror
  if (L >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_int(x), __float_as_int(x), false, false);
    x = op(__int_as_float(r[0]), __int_as_float(r[1]));
  }
  if (L >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_int(x), __float_as_int(x), false, false);
    x = op(__int_as_float(r[0]), __int_as_float(r[1]));
  }
  return x;
}
template <int L>
__device__ __forceinline__ float group_sum(float x) {
  return group_reduce<L>(x, [](float a, float b) { return a + b; });
}
template <int L>
__device__ __forceinline__ float group_max(float x) {
  return group_reduce<L>(x, [](float a, float b) { return fmaxf(a, b); });
}

// ---------------------------------------------------------------------------
// Softmax rows of router logits. L lanes hold a token's row of E <= 4 L logits,
// four consecutive experts each, so a wave works on 64 / L tokens at once and a
// row is read as one run of 16-byte loads. A block of 4 waves takes kRowIters
// rounds of them, all within one group (a sequence, or the whole batch).
// ---------------------------------------------------------------------------
constexpr int kRowIters = 8;

struct RowArgs {
  const float* z;        // [T, E]
  const int32_t* ids;    // [T, k]
  const uint8_t* mask;   // [T] or nullptr
  int T, E, k;
  int n;                 // tokens of a group
  int groups, blocks;    // groups, blocks of a group
};

// Four logits of a row, -inf past the last expert.
__device__ __forceinline__ float4 load_logits(const float* row, int e0, int E, bool vec, bool live) {
  const float ninf = -__builtin_huge_valf();
  float4 v = make_float4(ninf, ninf, ninf, ninf);
  if (!live) return v;
  if (vec) {
    if (e0 < E) v = *reinterpret_cast<const float4*>(row + e0);
  } else {
    if (e0 < E) v.x = row[e0];
    if (e0 + 1 < E) v.y = row[e0 + 1];
    if (e0 + 2 < E) v.z = row[e0 + 2];
    if (e0 + 3 < E) v.w = row[e0 + 3];
  }
  return v;
}

// exp(z - max z) of the row in v, and 1 / sum and the logarithm of the sum of
// exponentials. A row of -inf alone has no distribution: all three are 0.
template <int L>
__device__ __forceinline__ void row_softmax(float4& v, float& inv, float& lse) {
  const float top = group_max<L>(fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)));
  // a NaN is not the maximum of a row, but makes its sum a NaN
  const bool none = top == -__builtin_huge_valf();
  const float m = none ? 0.0f : top;
  v = make_float4(expf(v.x - m), expf(v.y - m), expf(v.z - m), expf(v.w - m));
  const float sum = group_sum<L>((v.x + v.y) + (v.z + v.w));
  const bool empty = sum == 0.0f;
  inv = empty ? 0.0f : 1.0f / sum;
  lse = empty ? 0.0f : m + logf(sum);
}

// ---------------------------------------------------------------------------
// Balance loss. With f_e = E c_e / (k n_s) and P_e = sum_t p_te / n_s of group s,
//   sum_e f_e P_e = E / (k n_s^2) sum_t sum_e c_e p_te,
// so once the counts are known, one pass over the logits gives a number per
// token, and no [E] sums have to be joined across blocks. The counts are integer
// sums, the losses are joined by the last block in block order: results do not
// depend on timing.
//
// ws: counts [groups][E], live tokens [groups] and a ticket, then two partial sums
// per block. All of it is zero before and after a call, whatever the sizes, so
// that calls of other sizes, whose parts lie elsewhere, can share it.
// ---------------------------------------------------------------------------
struct LossWs {
  int32_t* counts;
  int32_t* live;
  int32_t* ticket;
  float2* part;
};

constexpr int kCountIds = 4096;  // ids that a counting block takes

// Counts of a part of a group's ids: blocks (part, group).
__global__ __launch_bounds__(256) void balance_count_kernel(RowArgs a, LossWs ws) {
  __shared__ int32_t s_cnt[kMaxExperts];
  __shared__ int32_t s_live;
  const int tid = threadIdx.x;
  for (int g = blockIdx.y; g < a.groups; g += gridDim.y) {
    for (int e = tid; e < a.E; e += 256) s_cnt[e] = 0;
    if (tid == 0) s_live = 0;
    __syncthreads();
    const int tok = kCountIds / a.k;  // tokens of a part
    const int t0 = blockIdx.x * tok, t1 = min(t0 + tok, a.n);
    for (int t = t0 + tid; t < t1; t += 256) {
      const size_t row = (size_t)g * a.n + t;
      if (a.mask != nullptr && a.mask[row] == 0) continue;
      atomicAdd(&s_live, 1);
      for (int j = 0; j < a.k; ++j) {
        const int e = a.ids[row * a.k + j];
        if ((unsigned)e < (unsigned)a.E) atomicAdd(&s_cnt[e], 1);
      }
    }
    __syncthreads();
    for (int e = tid; e < a.E; e += 256)
      if (s_cnt[e] != 0) atomicAdd(ws.counts + (size_t)g * a.E + e, s_cnt[e]);
    if (tid == 0 && s_live != 0) atomicAdd(ws.live + g, s_live);
    __syncthreads();
  }
}

// E / (k n_s^2) of a group of n_s live tokens.
__device__ __forceinline__ float group_factor(int E, int k, int live) {
  return live > 0 ? (float)((double)E / ((double)k * live * live)) : 0.0f;
}

template <int L>
__global__ __launch_bounds__(256) void balance_loss_kernel(RowArgs a, LossWs ws, float* __restrict__ loss,
                                                           int32_t* __restrict__ counts, int32_t* __restrict__ live) {
  constexpr int SLOTS = kWave / L;
  __shared__ float2 s_part[4];
  __shared__ int s_last;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int g = (int)(blockIdx.x / a.blocks), blk = (int)(blockIdx.x - (unsigned)g * a.blocks);
  const int e0 = (lane % L) * 4;
  const bool vec = (a.E & 3) == 0;
  const float factor = group_factor(a.E, a.k, ws.live[g]);
  float c[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) c[q] = e0 + q < a.E ? (float)ws.counts[(size_t)g * a.E + e0 + q] : 0.0f;
  float bal = 0.0f, zl = 0.0f;
  float4 v[kRowIters];
  bool on[kRowIters];
#pragma unroll
  for (int i = 0; i < kRowIters; ++i) {
    const int t = (blk * kRowIters + i) * 4 * SLOTS + wave * SLOTS + lane / L;
    const size_t row = (size_t)g * a.n + t;
    on[i] = t < a.n && (a.mask == nullptr || a.mask[row] != 0);
    v[i] = load_logits(a.z + row * a.E, e0, a.E, vec, on[i]);
  }
#pragma unroll
  for (int i = 0; i < kRowIters; ++i) {
    float inv, lse;
    row_softmax<L>(v[i], inv, lse);
    const float s = group_sum<L>((c[0] * v[i].x + c[1] * v[i].y) + (c[2] * v[i].z + c[3] * v[i].w)) * inv;
    if (on[i] && lane % L == 0) bal += s, zl += lse * lse;
  }
  bal = group_sum<64>(bal);
  zl = group_sum<64>(zl);
  if (lane == 0) s_part[wave] = make_float2(bal, zl);
  __syncthreads();
  if (tid == 0) {
    float2 p = make_float2(0.0f, 0.0f);
    for (int w = 0; w < 4; ++w) p.x += s_part[w].x, p.y += s_part[w].y;
    // the block's part of its group's balance loss and of the z sum, in agent
    // scope: the last block runs on any XCD
    uint64_t u = (uint64_t)__float_as_uint(p.x * factor) | (uint64_t)__float_as_uint(p.y) << 32;
    __hip_atomic_store(reinterpret_cast<uint64_t*>(ws.part + blockIdx.x), u, __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
    s_last = __hip_atomic_fetch_add(ws.ticket, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
  }
  __syncthreads();
  if (!s_last) return;

  // The last block: every other one has read the counts. It hands them out,
  // clears them for the next call and joins the partial sums.
  double sb = 0.0, sz = 0.0;
  long long many = 0, full = 0;
  for (size_t i = tid; i < gridDim.x; i += 256) {
    const uint64_t u = __hip_atomic_load(reinterpret_cast<uint64_t*>(ws.part + i), __ATOMIC_RELAXED,
                                         __HIP_MEMORY_SCOPE_AGENT);
    sb += (double)__uint_as_float((uint32_t)u), sz += (double)__uint_as_float((uint32_t)(u >> 32));
    ws.part[i] = make_float2(0.0f, 0.0f);
  }
  for (size_t i = tid; i < (size_t)a.groups * a.E; i += 256) {
    counts[i] = ws.counts[i];
    ws.counts[i] = 0;
  }
  for (int i = tid; i < a.groups; i += 256) {
    const int n = ws.live[i];
    live[i] = n;
    ws.live[i] = 0;
    many += n, full += n > 0;
  }
  __shared__ double s_d[256][2];
  __shared__ long long s_n[256][2];
  s_d[tid][0] = sb, s_d[tid][1] = sz, s_n[tid][0] = many, s_n[tid][1] = full;
  __syncthreads();
  for (int w = 128; w > 0; w >>= 1) {
    if (tid < w)
#pragma unroll
      for (int q = 0; q < 2; ++q) s_d[tid][q] += s_d[tid + w][q], s_n[tid][q] += s_n[tid + w][q];
    __syncthreads();
  }
  if (tid == 0) {
    many = s_n[0][0], full = s_n[0][1];
    loss[0] = full > 0 ? (float)(s_d[0][0] / (double)full) : 0.0f;
    loss[1] = many > 0 ? (float)(s_d[0][1] / (double)many) : 0.0f;
    live[a.groups] = (int32_t)many;
    live[a.groups + 1] = (int32_t)full;
    *ws.ticket = 0;
  }
}

static int lanes_of(int E) {
  int L = 1;
  while (4 * L < E) L *= 2;
  return L;
}

// n > 0 tokens a group
static RowArgs row_args(const float* z, const int32_t* ids, const uint8_t* mask, int T, int E, int k, int n) {
  RowArgs a{z, ids, mask, T, E, k, n, T / n, 0};
  const int per = kRowIters * 4 * (kWave / lanes_of(E));
  a.blocks = (n + per - 1) / per;
  return a;
}

static size_t round256(size_t n) { return (n + 255) / 256 * 256; }

long long balance_blocks(int T, int E, int n) {
  if (T == 0) return 0;
  const RowArgs a = row_args(nullptr, nullptr, nullptr, T, E, 1, n);
  return (long long)a.groups * a.blocks;
}

size_t balance_ws_bytes(int T, int E, int k, int n) {
  if (T == 0) return 256;
  const RowArgs a = row_args(nullptr, nullptr, nullptr, T, E, k, n);
  return round256((size_t)a.groups * E * 4) + round256(((size_t)a.groups + 1) * 4) +
         round256((size_t)a.groups * a.blocks * 8);
}

// launch(std::integral_constant) for the lanes a row of E logits takes
template <class Launch>
static void by_lanes(int E, Launch&& launch) {
  switch (lanes_of(E)) {
    case 1: launch(std::integral_constant<int, 1>()); break;
    case 2: launch(std::integral_constant<int, 2>()); break;
    case 4: launch(std::integral_constant<int, 4>()); break;
    case 8: launch(std::integral_constant<int, 8>()); break;
    case 16: launch(std::integral_constant<int, 16>()); break;
    case 32: launch(std::integral_constant<int, 32>()); break;
    default: launch(std::integral_constant<int, 64>()); break;
  }
}

// No tokens: `groups` groups (one or none) without any.
__global__ void balance_empty_kernel(int groups, int E, float* loss, int32_t* counts, int32_t* live) {
  for (int i = threadIdx.x; i < groups * E; i += 256) counts[i] = 0;
  if (threadIdx.x < 2) loss[threadIdx.x] = 0.0f;
  for (int i = threadIdx.x; i < groups + 2; i += 256) live[i] = 0;
}

hipError_t launch_balance_empty(int groups, int E, float* loss, int32_t* counts, int32_t* live, hipStream_t s) {
  balance_empty_kernel<<<1, 256, 0, s>>>(groups, E, loss, counts, live);
  return hipGetLastError();
}

hipError_t launch_balance_loss(const float* z, const int32_t* ids, const uint8_t* mask, int T, int E, int k, int n,
                               float* loss, int32_t* counts, int32_t* live, void* wsp, hipStream_t s) {
  const RowArgs a = row_args(z, ids, mask, T, E, k, n);
  char* w = static_cast<char*>(wsp);
  LossWs ws;
  ws.counts = reinterpret_cast<int32_t*>(w);
  w += round256((size_t)a.groups * E * 4);
  ws.live = reinterpret_cast<int32_t*>(w);
  ws.ticket = ws.live + a.groups;
  w += round256(((size_t)a.groups + 1) * 4);
  ws.part = reinterpret_cast<float2*>(w);
  const int tok = kCountIds / k;
  balance_count_kernel<<<dim3((unsigned)((n + tok - 1) / tok), (unsigned)std::min(a.groups, 4096)), 256, 0, s>>>(a, ws);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  by_lanes(E, [&](auto l) {
    balance_loss_kernel<decltype(l)::value><<<(unsigned)(a.groups * a.blocks), 256, 0, s>>>(a, ws, loss, counts, live);
  });
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Gradient to the logits. Of the losses, for a live token of group s,
//   g_b / S' E / (k n_s^2) p_e (c_e - sum_j c_j p_j) + g_z 2 / n lse p_e,
// and of the gate weights w = softmax of the selected logits, for every token,
//   w_j (dw_j - sum_i w_i dw_i) at expert ids_j.
// One pass: logits in, gradient out. The selected experts' terms reach the lanes
// that hold them through one row of LDS per token, which is zero between uses.
// ---------------------------------------------------------------------------
struct GateGradArgs {
  const int32_t* counts;   // [groups, E]
  const int32_t* live;     // [groups + 2]
  const float* dloss;      // [2]
  const float* w;          // [T, k] or nullptr
  const float* dw;         // [T, k]
  float* dz;               // [T, E]
};

template <int L>
__global__ __launch_bounds__(256) void gate_backward_kernel(RowArgs a, GateGradArgs b) {
  constexpr int SLOTS = kWave / L;
  __shared__ __align__(16) float s_row[4][SLOTS][L * 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane % L, slot = lane / L;
  const int g = (int)(blockIdx.x / a.blocks), blk = (int)(blockIdx.x - (unsigned)g * a.blocks);
  const int e0 = sub * 4;
  const bool vec = (a.E & 3) == 0;
  float4* mine = reinterpret_cast<float4*>(&s_row[wave][slot][e0]);
  *mine = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  const int many = b.live[a.groups], full = b.live[a.groups + 1];
  const float gb = full > 0 ? b.dloss[0] * group_factor(a.E, a.k, b.live[g]) / (float)full : 0.0f;
  const float gz = many > 0 ? b.dloss[1] * 2.0f / (float)many : 0.0f;
  float c[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) c[q] = e0 + q < a.E ? (float)b.counts[(size_t)g * a.E + e0 + q] : 0.0f;
  float4 v[kRowIters];
  bool on[kRowIters];
#pragma unroll
  for (int i = 0; i < kRowIters; ++i) {
    const int t = (blk * kRowIters + i) * 4 * SLOTS + wave * SLOTS + slot;
    const size_t row = (size_t)g * a.n + t;
    on[i] = t < a.n && (a.mask == nullptr || a.mask[row] != 0);
    v[i] = load_logits(a.z + row * a.E, e0, a.E, vec, on[i]);
  }
#pragma unroll
  for (int i = 0; i < kRowIters; ++i) {
    const int t = (blk * kRowIters + i) * 4 * SLOTS + wave * SLOTS + slot;
    const size_t row = (size_t)g * a.n + t;
    float inv, lse;
    row_softmax<L>(v[i], inv, lse);
    const float s = group_sum<L>((c[0] * v[i].x + c[1] * v[i].y) + (c[2] * v[i].z + c[3] * v[i].w)) * inv;
    const float zt = gz * lse;
    auto grad = [&](float ex, float ce) { return on[i] ? ex * inv * (gb * (ce - s) + zt) : 0.0f; };
    float4 d = make_float4(grad(v[i].x, c[0]), grad(v[i].y, c[1]), grad(v[i].z, c[2]), grad(v[i].w, c[3]));
    if (b.w != nullptr) {
      float dot = 0.0f;
      if (t < a.n)
        for (int j = sub; j < a.k; j += L) dot += b.w[row * a.k + j] * b.dw[row * a.k + j];
      dot = group_sum<L>(dot);
      if (t < a.n)
        for (int j = sub; j < a.k; j += L) {
          const int e = a.ids[row * a.k + j];
          if ((unsigned)e < (unsigned)a.E)
            atomicAdd(&s_row[wave][slot][e], b.w[row * a.k + j] * (b.dw[row * a.k + j] - dot));
        }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      const float4 add = *mine;
      *mine = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      d.x += add.x, d.y += add.y, d.z += add.z, d.w += add.w;
    }
    if (t < a.n) {
      float* out = b.dz + row * a.E;
      if (vec) {
        if (e0 < a.E) *reinterpret_cast<float4*>(out + e0) = d;
      } else {
        if (e0 < a.E) out[e0] = d.x;
        if (e0 + 1 < a.E) out[e0 + 1] = d.y;
        if (e0 + 2 < a.E) out[e0 + 2] = d.z;
        if (e0 + 3 < a.E) out[e0 + 3] = d.w;
      }
    }
  }
}

hipError_t launch_gate_backward(const float* z, const int32_t* ids, const uint8_t* mask, int T, int E, int k, int n,
                                const int32_t* counts, const int32_t* live, const float* dloss, const float* w,
                                const float* dw, float* dz, hipStream_t s) {
  const RowArgs a = row_args(z, ids, mask, T, E, k, n);
  const GateGradArgs b{counts, live, dloss, w, dw, dz};
  by_lanes(E, [&](auto l) {
    gate_backward_kernel<decltype(l)::value><<<(unsigned)(a.groups * a.blocks), 256, 0, s>>>(a, b);
  });
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Gradient of the combine out[t] = sum_j w_tj y[dest_tj]: dw_tj = <dout_t,
// y[dest_tj]> (0 for a remote assignment) and dy[dest_tj] = w_tj dout_t. One
// wave per token reads its dout row once and each of its expert rows once; fp32
// products and sums.
// ---------------------------------------------------------------------------
constexpr int kCombineGradVecs = 4;  // 16-byte pieces of a row per lane in flight

template <bool BF16>
__global__ __launch_bounds__(256) void combine_backward_kernel(const uint4* __restrict__ dout,
                                                               const uint4* __restrict__ y,
                                                               const float* __restrict__ w,
                                                               const int32_t* __restrict__ dest, int T, int k,
                                                               int row_vecs, int M_cap, float* __restrict__ dw,
                                                               uint4* __restrict__ dy) {
  constexpr int U = kCombineGradVecs, N = BF16 ? 8 : 4;
  const int lane = threadIdx.x & 63;
  const int t = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  if (t >= T) return;
  // assignment j sits in lane j
  int d = -1;
  float wt = 0.0f;
  if (lane < k) {
    d = dest[(size_t)t * k + lane];
    if (d >= M_cap) d = -1;
    wt = w[(size_t)t * k + lane];
  }
  const uint64_t local = __ballot(d >= 0);
  float mine = 0.0f;  // lane j's dw
  if (local != 0) {
    float acc[kMaxTopk];
#pragma unroll
    for (int j = 0; j < kMaxTopk; ++j) acc[j] = 0.0f;
    auto unpack = [](uint4 u, float (&f)[N]) {
      const uint32_t q[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (BF16) {
          f[2 * i] = __uint_as_float(q[i] << 16);
          f[2 * i + 1] = __uint_as_float(q[i] & 0xffff0000u);
        } else {
          f[i] = __uint_as_float(q[i]);
        }
      }
    };
    for (int v0 = 0; v0 < row_vecs; v0 += U * kWave) {
      uint4 g[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int v = v0 + u * kWave + lane;
        g[u] = v < row_vecs ? dout[(size_t)t * row_vecs + v] : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int j = 0; j < kMaxTopk; ++j) {
        if (j >= k || !((local >> j) & 1)) continue;
        const int dj = __builtin_amdgcn_readlane(d, j);
        const float wj = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(wt), j));
        uint4 yv[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int v = v0 + u * kWave + lane;
          yv[u] = v < row_vecs ? y[(size_t)dj * row_vecs + v] : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int v = v0 + u * kWave + lane;
          float a[N], b[N];
          unpack(g[u], a);
          unpack(yv[u], b);
          float s = 0.0f;
#pragma unroll
          for (int i = 0; i < N; ++i) s = fmaf(a[i], b[i], s);
          acc[j] += s;
          if (dy != nullptr && v < row_vecs) {
            uint4 o;
            if constexpr (BF16)
              o = make_uint4(pack_bf16x2(wj * a[0], wj * a[1]), pack_bf16x2(wj * a[2], wj * a[3]),
                             pack_bf16x2(wj * a[4], wj * a[5]), pack_bf16x2(wj * a[6], wj * a[7]));
            else
              o = make_uint4(__float_as_uint(wj * a[0]), __float_as_uint(wj * a[1]), __float_as_uint(wj * a[2]),
                             __float_as_uint(wj * a[3]));
            dy[(size_t)dj * row_vecs + v] = o;
          }
        }
      }
    }
#pragma unroll
    for (int j = 0; j < kMaxTopk; ++j) {
      if (j >= k || !((local >> j) & 1)) continue;
      const float s = group_sum<64>(acc[j]);
      if (lane == j) mine = s;
    }
  }
  if (lane < k) dw[(size_t)t * k + lane] = mine;
}

hipError_t launch_combine_backward(const void* dout, const void* y, const float* w, const int32_t* dest, int T, int k,
                                   int H, int M_cap, bool bf16, float* dw, void* dy, hipStream_t s) {
  const unsigned grid = (unsigned)((T + 3) / 4);
  if (bf16)
    combine_backward_kernel<true><<<grid, 256, 0, s>>>(static_cast<const uint4*>(dout), static_cast<const uint4*>(y),
                                                       w, dest, T, k, H / 8, M_cap, dw, static_cast<uint4*>(dy));
  else
    combine_backward_kernel<false><<<grid, 256, 0, s>>>(static_cast<const uint4*>(dout),
                                                        static_cast<const uint4*>(y), w, dest, T, k, H / 4, M_cap, dw,
                                                        static_cast<uint4*>(dy));
  return hipGetLastError();
}

}  // namespace moe
