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
// row is read as one run of 16-byte loads. A block of W waves takes N rounds of
// them, all within one group (a sequence, or the whole batch), with the loads of all
// rounds in flight before the first is used. N is small: each launch fetches its code
// from beyond the L2, and long unrolled code costs more than it hides.
//
// Exponentials and logarithms are the hardware's base-2 ones (1 ulp): with the
// rounding of (z - max) log2 e, |z - max| 2^-24 relative in p.
// ---------------------------------------------------------------------------
static int lanes_of(int E) {
  int L = 1;
  while (4 * L < E) L *= 2;
  return L;
}

struct RowArgs {
  const float* z;        // [T, E]
  const int32_t* ids;    // [T, k]
  const uint8_t* mask;   // [T] or nullptr
  int T, E, k;
  int n;                 // tokens of a group
  int groups, blocks;    // groups, blocks of a group
};

// Four logits of a row, -inf past the last expert.
__device__ __forceinline__ float4 load_logits(const float* row, int e0, int E, bool vec, bool in) {
  const float ninf = -__builtin_huge_valf();
  float4 v = make_float4(ninf, ninf, ninf, ninf);
  if (!in) return v;
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

// The rows of a block: this lane's logits of every round, and whether the token
// is there (in) and live (on). Masked rows are read as well, so that the loads
// wait for nothing; settle, which waits for them, replaces what they hold by -inf.
template <int L, int W, int N>
struct Rows {
  float4 v[N];
  bool in[N], on[N];
  size_t row[N];
  uint8_t m[N];

  // rounds [first, first + N) of block blk's `rounds`
  __device__ __forceinline__ void load(const RowArgs& a, int g, int blk, int rounds, int first, int lane, int wave) {
    constexpr int SLOTS = kWave / L;
    const int e0 = (lane % L) * 4;
    const bool vec = (a.E & 3) == 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int t = (blk * rounds + first + i) * W * SLOTS + wave * SLOTS + lane / L;
      in[i] = t < a.n;
      row[i] = (size_t)g * a.n + (in[i] ? t : 0);
      v[i] = load_logits(a.z + row[i] * a.E, e0, a.E, vec, in[i]);
      m[i] = a.mask != nullptr ? a.mask[row[i]] : 1;
    }
  }
  __device__ __forceinline__ void settle() {
    const float ninf = -__builtin_huge_valf();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      on[i] = in[i] && m[i] != 0;
      if (!on[i]) v[i] = make_float4(ninf, ninf, ninf, ninf);
    }
  }
};

// exp(z - max z) of the row in v, and 1 / sum and the logarithm of the sum of
// exponentials. A row of -inf alone has no distribution: all three are 0.
template <int L>
__device__ __forceinline__ void row_softmax(float4& v, float& inv, float& lse) {
  const float top = group_max<L>(fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)));
  // a NaN is not the maximum of a row, but makes its sum a NaN
  const float m = top == -__builtin_huge_valf() ? 0.0f : top;
  auto ex = [&](float z) { return __builtin_amdgcn_exp2f((z - m) * 1.4426950408889634f); };
  v = make_float4(ex(v.x), ex(v.y), ex(v.z), ex(v.w));
  const float sum = group_sum<L>((v.x + v.y) + (v.z + v.w));
  const bool empty = sum == 0.0f;
  inv = empty ? 0.0f : __builtin_amdgcn_rcpf(sum);
  lse = empty ? 0.0f : m + __builtin_amdgcn_logf(sum) * 0.6931471805599453f;
}

// ---------------------------------------------------------------------------
// Balance loss. With f_e = E c_e / (k n_s) and P_e = sum_t p_te / n_s of group s,
//   sum_e f_e P_e = E / (k n_s^2) sum_t sum_e c_e p_te,
// so once the counts are known, one pass over the logits gives a number per
// token, and no [E] sums have to be joined across blocks. The counts are integer
// sums, the losses are joined by the last block in block order: results do not
// depend on timing. A group of at most kSelfIds ids is counted by each of its
// blocks itself, which saves the counting launch; a larger one in up to kParts
// parts first, whose counts each block adds up (no atomics: 8192 of them on 1024
// counters took 9 us).
//
// 16384 tokens of 256 experts in 4 groups (16.8 MB of logits): counts 6.2 us, loss 11 to
// 13, where the copy rate alone would take 4: a launch, counts, logits and the join
// follow each other, each a latency. 64 tokens of 8 experts in one launch of 5.4 us.
//
// ws: a ticket, zero before and after a call (at the start, whatever the sizes), two
// partial sums per block, the counts and live tokens of the parts.
// ---------------------------------------------------------------------------
struct LossWs {
  int32_t* ticket;
  uint64_t* part;   // [blocks]
  int32_t* counts;  // [groups][parts][4 L]
  int32_t* live;    // [groups][parts]
  int parts;        // 0: a block counts its group itself
};

constexpr int kSelfIds = 4096;
constexpr int kParts = 32;

// Adds the ids of tokens [t0, t1) of group g that are live to cnt[E] and their
// number to live (LDS), a token per thread.
template <int THREADS>
__device__ __forceinline__ void count_ids(const RowArgs& a, int g, int t0, int t1, int32_t* cnt, int32_t* live) {
  constexpr int IDS = 8;  // ids of a token in flight
  const int k = a.k;
  int n = 0;
  for (int t = t0 + (int)threadIdx.x; t < t1; t += THREADS) {
    const size_t row = (size_t)g * a.n + t;
    const uint8_t m = a.mask != nullptr ? a.mask[row] : 1;
#pragma unroll 1
    for (int j0 = 0; j0 < k; j0 += IDS) {
      int e[IDS];
#pragma unroll
      for (int j = 0; j < IDS; ++j) e[j] = a.ids[row * k + min(j0 + j, k - 1)];
#pragma unroll
      for (int j = 0; j < IDS; ++j)
        if (m != 0 && j0 + j < k && (unsigned)e[j] < (unsigned)a.E) atomicAdd(cnt + e[j], 1);
    }
    n += m != 0;
  }
  if (n > 0) atomicAdd(live, n);
}

// Counts of part blockIdx.x of a group's tokens.
__global__ __launch_bounds__(256) void balance_count_kernel(RowArgs a, LossWs ws, int ep, int tok) {
  __shared__ int32_t s_cnt[kMaxExperts];
  __shared__ int32_t s_live;
  const int tid = threadIdx.x, p = blockIdx.x;
  // less than 2^31 (as count_ids' steps past t1 are): n <= 2^31 - 256 (moe_abi.cpp)
  const int t0 = min(p * tok, a.n), t1 = min(t0 + tok, a.n);
  for (int g = blockIdx.y; g < a.groups; g += gridDim.y) {
    s_cnt[tid] = 0;
    if (tid == 0) s_live = 0;
    __syncthreads();
    count_ids<256>(a, g, t0, t1, s_cnt, &s_live);
    __syncthreads();
    const size_t at = (size_t)g * ws.parts + p;
    if (tid < ep) ws.counts[at * ep + tid] = s_cnt[tid];
    if (tid == 0) ws.live[at] = s_live;
    __syncthreads();
  }
}

// E / (k n_s^2) of a group of n_s live tokens.
__device__ __forceinline__ float group_factor(int E, int k, int live) {
  return live > 0 ? (float)((double)E / ((double)k * live * live)) : 0.0f;
}

constexpr int kLossWaves = 8, kLossRounds = 8;  // of a block; kLossFlight rounds in flight
constexpr int kLossFlight = 4;

template <int L, bool SELF>
__global__ __launch_bounds__(kLossWaves* kWave) void balance_loss_kernel(RowArgs a, LossWs ws, float* __restrict__ loss,
                                                           int32_t* __restrict__ counts, int32_t* __restrict__ live) {
  constexpr int W = kLossWaves, N = kLossFlight, THREADS = W * kWave;
  __shared__ float2 s_part[W];
  __shared__ int s_last;
  __shared__ __align__(16) int32_t s_cnt[kMaxExperts];
  __shared__ int32_t s_live;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int g = (int)(blockIdx.x / a.blocks), blk = (int)(blockIdx.x - (unsigned)g * a.blocks);
  const int e0 = (lane % L) * 4;
  Rows<L, W, N> r;
  r.load(a, g, blk, kLossRounds, 0, lane, wave);
  if (tid < kMaxExperts) s_cnt[tid] = 0;
  if (tid == 0) s_live = 0;
  __syncthreads();
  if (SELF) {
    count_ids<THREADS>(a, g, 0, a.n, s_cnt, &s_live);
  } else {
    // four counts of a part at a time, all of a thread's in flight
    constexpr int C = (kParts * L + THREADS - 1) / THREADS;
    const int4* parts = reinterpret_cast<const int4*>(ws.counts + (size_t)g * ws.parts * (4 * L));
    int4 q[C];
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int at = i * THREADS + tid;
      q[i] = at < ws.parts * L ? parts[at] : make_int4(0, 0, 0, 0);
    }
    const int n = tid < ws.parts ? ws.live[(size_t)g * ws.parts + tid] : 0;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      int32_t* s = s_cnt + ((i * THREADS + tid) % L) * 4;
      if (q[i].x) atomicAdd(s, q[i].x);
      if (q[i].y) atomicAdd(s + 1, q[i].y);
      if (q[i].z) atomicAdd(s + 2, q[i].z);
      if (q[i].w) atomicAdd(s + 3, q[i].w);
    }
    if (n != 0) atomicAdd(&s_live, n);
  }
  __syncthreads();
  const int n_live = s_live;
  const int4 n4 = *reinterpret_cast<const int4*>(s_cnt + e0);  // of this lane's experts
  const float c[4] = {(float)n4.x, (float)n4.y, (float)n4.z, (float)n4.w};
  if (blk == 0 && tid < L) {
    int32_t* out = counts + (size_t)g * a.E + e0;
    if (e0 < a.E) out[0] = n4.x;
    if (e0 + 1 < a.E) out[1] = n4.y;
    if (e0 + 2 < a.E) out[2] = n4.z;
    if (e0 + 3 < a.E) out[3] = n4.w;
    if (tid == 0) __hip_atomic_store(live + g, n_live, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  float bal = 0.0f, zl = 0.0f;
#pragma unroll 1
  for (int first = 0;;) {
    // the next rounds' loads leave before these are used
    first += N;
    const bool more = first < kLossRounds && (blk * kLossRounds + first) * W * (kWave / L) < a.n;
    Rows<L, W, N> next;
    if (more) next.load(a, g, blk, kLossRounds, first, lane, wave);
    r.settle();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float4& v = r.v[i];
      float inv, lse;
      row_softmax<L>(v, inv, lse);
      const float s = group_sum<L>((c[0] * v.x + c[1] * v.y) + (c[2] * v.z + c[3] * v.w)) * inv;
      if (r.on[i] && lane % L == 0) bal += s, zl += lse * lse;
    }
    if (!more) break;
    r = next;
  }
  bal = group_sum<64>(bal);
  zl = group_sum<64>(zl);
  if (lane == 0) s_part[wave] = make_float2(bal, zl);
  __syncthreads();
  const float factor = group_factor(a.E, a.k, n_live);
  double sb = 0.0, sz = 0.0;
  int many = 0, full = 0;  // at most T each
  if (gridDim.x == 1) {    // nothing to join
    if (tid != 0) return;
    for (int w = 0; w < W; ++w) sb += s_part[w].x, sz += s_part[w].y;
    sb *= factor, many = n_live, full = n_live > 0;
  } else {
    if (tid == 0) {
      float2 p = make_float2(0.0f, 0.0f);
      for (int w = 0; w < W; ++w) p.x += s_part[w].x, p.y += s_part[w].y;
      // the block's part of its group's balance loss and of the z sum, written
      // through to where the last block, on any XCD, reads it, and there before the
      // ticket is drawn (no fence: that would write back the XCD's whole L2)
      const uint64_t u = (uint64_t)__float_as_uint(p.x * factor) | (uint64_t)__float_as_uint(p.y) << 32;
      __hip_atomic_store(ws.part + blockIdx.x, u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      wait_vmcnt<0>();
      s_last = __hip_atomic_fetch_add(ws.ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (int)gridDim.x - 1;
    }
    __syncthreads();
    if (!s_last) return;
    // The last block joins the sums and puts the ticket back.
    for (size_t i = tid; i < gridDim.x; i += THREADS) {
      const uint64_t u = __hip_atomic_load(ws.part + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      sb += (double)__uint_as_float((uint32_t)u), sz += (double)__uint_as_float((uint32_t)(u >> 32));
    }
    for (int i = tid; i < a.groups; i += THREADS) {
      const int n = __hip_atomic_load(live + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      many += n, full += n > 0;
    }
    __shared__ double s_d[THREADS][2];
    __shared__ int2 s_n[THREADS];
    s_d[tid][0] = sb, s_d[tid][1] = sz, s_n[tid] = make_int2(many, full);
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int q = 1; q < W; ++q) {
      sb += s_d[tid + 64 * q][0], sz += s_d[tid + 64 * q][1];
      many += s_n[tid + 64 * q].x, full += s_n[tid + 64 * q].y;
    }
#pragma unroll
    for (int w = 32; w > 0; w >>= 1) {
      sb += __shfl_xor(sb, w, kWave), sz += __shfl_xor(sz, w, kWave);
      many += __shfl_xor(many, w, kWave), full += __shfl_xor(full, w, kWave);
    }
    if (tid == 0) *ws.ticket = 0;
  }
  if (tid == 0) {
    loss[0] = full > 0 ? (float)(sb / (double)full) : 0.0f;
    loss[1] = many > 0 ? (float)(sz / (double)many) : 0.0f;
    live[a.groups] = many;
    live[a.groups + 1] = full;
  }
}

// Tokens of a block of the two kernels that read the logits.
static int loss_rows(int E) { return kLossWaves * kLossRounds * (kWave / lanes_of(E)); }
static int gate_rows(int E);

// n > 0 tokens a group
static RowArgs row_args(const float* z, const int32_t* ids, const uint8_t* mask, int T, int E, int k, int n,
                        int rows) {
  return {z, ids, mask, T, E, k, n, T / n, (n - 1) / rows + 1};
}

static size_t round256(size_t n) { return (n + 255) / 256 * 256; }

long long balance_blocks(int T, int E, int n) {
  if (T == 0) return 0;
  const RowArgs a = row_args(nullptr, nullptr, nullptr, T, E, 1, n, gate_rows(E));
  return (long long)a.groups * a.blocks;  // the loss has no more
}

// Parts that a group's ids are counted in; 0: by each block.
static int count_parts(int n, int k) {
  const long long ids = (long long)n * k;
  return ids <= kSelfIds ? 0 : (int)std::min<long long>(kParts, (ids + 2047) / 2048);
}

static LossWs loss_ws(const RowArgs& a, void* base, size_t* bytes) {
  LossWs ws;
  char* w = static_cast<char*>(base);
  ws.parts = count_parts(a.n, a.k);
  ws.ticket = reinterpret_cast<int32_t*>(w);
  size_t at = 256;
  ws.part = reinterpret_cast<uint64_t*>(w + at);
  at += round256((size_t)a.groups * a.blocks * 8);
  ws.counts = reinterpret_cast<int32_t*>(w + at);
  at += round256((size_t)a.groups * ws.parts * 4 * lanes_of(a.E) * 4);
  ws.live = reinterpret_cast<int32_t*>(w + at);
  at += round256((size_t)a.groups * ws.parts * 4);
  *bytes = at;
  return ws;
}

size_t balance_ws_bytes(int T, int E, int k, int n) {
  size_t bytes = 256;
  if (T > 0) (void)loss_ws(row_args(nullptr, nullptr, nullptr, T, E, k, n, loss_rows(E)), nullptr, &bytes);
  return bytes;
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
  const RowArgs a = row_args(z, ids, mask, T, E, k, n, loss_rows(E));
  size_t bytes;
  const LossWs ws = loss_ws(a, wsp, &bytes);
  const bool self = ws.parts == 0;
  if (!self) {
    balance_count_kernel<<<dim3((unsigned)ws.parts, (unsigned)std::min(a.groups, 65535)), 256, 0, s>>>(
        a, ws, 4 * lanes_of(E), (n - 1) / ws.parts + 1);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  by_lanes(E, [&](auto l) {
    constexpr int L = decltype(l)::value;
    const unsigned grid = (unsigned)(a.groups * a.blocks);
    if (self)
      balance_loss_kernel<L, true><<<grid, kLossWaves * kWave, 0, s>>>(a, ws, loss, counts, live);
    else
      balance_loss_kernel<L, false><<<grid, kLossWaves * kWave, 0, s>>>(a, ws, loss, counts, live);
  });
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Gradient to the logits. Of the losses, for a live token of group s,
//   g_b / S' E / (k n_s^2) p_e (c_e - sum_j c_j p_j) + g_z 2 / n lse p_e,
// and of the gate weights w = softmax of the selected logits, for every token,
//   w_j (dw_j - sum_i w_i dw_i) at expert ids_j.
// One pass: logits in, gradient out. The selected experts' terms reach the lanes
// that hold them through one row of LDS per token, which is zero between uses. 16384
// tokens of 256 experts, top 8 (35 MB): 11-12 us, 3 TB/s, bound by the launch's
// ramp, one round of load latencies and the stores.
// ---------------------------------------------------------------------------
struct GateGradArgs {
  const int32_t* counts;   // [groups, E]
  const int32_t* live;     // [groups + 2]
  const float* dloss;      // [2]
  const float* w;          // [T, k] or nullptr
  const float* dw;         // [T, k]
  float* dz;               // [T, E]
};

// Rounds of a block of 4 waves: few where a lane has many of a token's top-k.
static constexpr int gate_rounds(int L) { return L >= 16 ? 4 : (L >= 4 ? 2 : 1); }
static int gate_rows(int E) { return gate_rounds(lanes_of(E)) * 4 * (kWave / lanes_of(E)); }

template <int L, bool GATE>
__global__ __launch_bounds__(256) void gate_backward_kernel(RowArgs a, GateGradArgs b) {
  constexpr int SLOTS = kWave / L, N = gate_rounds(L), PL = (kMaxTopk + L - 1) / L;
  __shared__ __align__(16) float s_row[GATE ? 4 : 1][SLOTS][L * 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane % L, slot = lane / L;
  const int g = (int)(blockIdx.x / a.blocks), blk = (int)(blockIdx.x - (unsigned)g * a.blocks);
  const int e0 = sub * 4;
  const bool vec = (a.E & 3) == 0;
  Rows<L, 4, N> r;
  r.load(a, g, blk, N, 0, lane, wave);
  float w[N][PL], dw[N][PL];
  int id[N][PL];
  if (GATE) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int q = 0; q < PL; ++q) {
        const int j = q * L + sub;
        const bool there = r.in[i] && j < a.k;
        const size_t at = there ? r.row[i] * a.k + j : 0;
        w[i][q] = there ? b.w[at] : 0.0f;
        dw[i][q] = there ? b.dw[at] : 0.0f;
        id[i][q] = there ? a.ids[at] : -1;
      }
  }
  const int many = b.live[a.groups], full = b.live[a.groups + 1];
  const float gb = full > 0 ? b.dloss[0] * group_factor(a.E, a.k, b.live[g]) / (float)full : 0.0f;
  const float gz = many > 0 ? b.dloss[1] * 2.0f / (float)many : 0.0f;
  float c[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) c[q] = e0 + q < a.E ? (float)b.counts[(size_t)g * a.E + e0 + q] : 0.0f;
  float* srow = s_row[GATE ? wave : 0][slot];
  float4* mine = reinterpret_cast<float4*>(srow + e0);
  if (GATE) *mine = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  r.settle();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    float4& v = r.v[i];
    float inv, lse;
    row_softmax<L>(v, inv, lse);
    const float s = group_sum<L>((c[0] * v.x + c[1] * v.y) + (c[2] * v.z + c[3] * v.w)) * inv;
    const float zt = gz * lse;
    auto grad = [&](float ex, float ce) { return r.on[i] ? ex * inv * (gb * (ce - s) + zt) : 0.0f; };
    float4 d = make_float4(grad(v.x, c[0]), grad(v.y, c[1]), grad(v.z, c[2]), grad(v.w, c[3]));
    if (GATE) {
      float dot = 0.0f;
#pragma unroll
      for (int q = 0; q < PL; ++q) dot += w[i][q] * dw[i][q];
      dot = group_sum<L>(dot);
#pragma unroll
      for (int q = 0; q < PL; ++q)
        if ((unsigned)id[i][q] < (unsigned)a.E) atomicAdd(srow + id[i][q], w[i][q] * (dw[i][q] - dot));
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      const float4 add = *mine;
      *mine = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      d.x += add.x, d.y += add.y, d.z += add.z, d.w += add.w;
    }
    if (r.in[i]) {
      float* out = b.dz + r.row[i] * a.E;
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
  const RowArgs a = row_args(z, ids, mask, T, E, k, n, gate_rows(E));
  const GateGradArgs b{counts, live, dloss, w, dw, dz};
  by_lanes(E, [&](auto l) {
    constexpr int L = decltype(l)::value;
    const unsigned grid = (unsigned)(a.groups * a.blocks);
    if (w != nullptr)
      gate_backward_kernel<L, true><<<grid, 256, 0, s>>>(a, b);
    else
      gate_backward_kernel<L, false><<<grid, 256, 0, s>>>(a, b);
  });
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Gradient of the combine out[t] = sum_j w_tj y[dest_tj]: dw_tj = <dout_t,
// y[dest_tj]> (0 for a remote assignment) and dy[dest_tj] = w_tj dout_t. One
// wave per token reads its dout row once and each of its expert rows once; fp32
// products and sums. Copy bound: 16384 tokens, a shard of 32 of 256 experts, H = 7168
// (630 MB) 132-135 us, 4.7 TB/s.
// ---------------------------------------------------------------------------
constexpr int kCombineGradVecs = 4;  // 16-byte pieces of a row per lane in flight
constexpr unsigned kCombineGradTokens = 1u << 25;  // of a launch

template <bool BF16>
__global__ __launch_bounds__(256) void combine_backward_kernel(const uint4* __restrict__ dout,
                                                               const uint4* __restrict__ y,
                                                               const float* __restrict__ w,
                                                               const int32_t* __restrict__ dest, int T, int k,
                                                               int row_vecs, int M_cap, float* __restrict__ dw,
                                                               uint4* __restrict__ dy, unsigned first) {
  constexpr int U = kCombineGradVecs, N = BF16 ? 8 : 4;
  const int lane = threadIdx.x & 63;
  const unsigned t = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)) + first;
  if (t >= (unsigned)T) return;
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
  // a launch has less than 2^32 threads: more than kCombineGradTokens tokens take several
  for (unsigned first = 0; first < (unsigned)T; first += kCombineGradTokens) {
    const unsigned grid = (std::min((unsigned)T - first, kCombineGradTokens) - 1) / 4 + 1;
    if (bf16)
      combine_backward_kernel<true><<<grid, 256, 0, s>>>(static_cast<const uint4*>(dout),
                                                         static_cast<const uint4*>(y), w, dest, T, k, H / 8, M_cap, dw,
                                                         static_cast<uint4*>(dy), first);
    else
      combine_backward_kernel<false><<<grid, 256, 0, s>>>(static_cast<const uint4*>(dout),
                                                          static_cast<const uint4*>(y), w, dest, T, k, H / 4, M_cap,
                                                          dw, static_cast<uint4*>(dy), first);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace moe
