// Grouped SwiGLU expert FFN (gfx950): the expert computation whose latency
// per token load is ViBE's per-GPU performance model f_g(n) (Section 4.2.1).
//
// Two persistent launches per call:
//   gate/up:  h[R] = bf16( silu(X_R W_gate^T) * (X_R W_up^T) )   (dual GEMM)
//   down:     y[R] = bf16( h[R] W_down^T )
// for each local expert's row range R = [offsets[e], offsets[e+1]), each
// followed by a small reduction that finishes split-K tiles (it returns at
// once when the GEMM split nothing).
//
// Per-expert row counts live only on the device, so each block rebuilds the
// tile list from `offsets` (a scan over at most 256 experts) and walks it
// with a grid stride. Rows are cut into 256-row tiles plus one 64-, 128- or
// 256-row remainder tile (row_tiles, tile_class). Within an expert,
// consecutive tile indices share a weight column block, so blocks running at
// the same time read the same weights.
#include <algorithm>
#include <mutex>

#include "common.hpp"
#include "grouped_gemm.hpp"
#include "launch.hpp"
#include "mx.hpp"

namespace moe {

template <bool DUAL, int W>
__global__ __launch_bounds__(W* kWave) void grouped_gemm_bf16_kernel(GemmArgs a) {
  grouped_gemm_body<W, DUAL, kBf16>(a);
}

// MXFP8 grouped GEMM: the same tile schedule; the dual GEMM writes MXFP8 h,
// the single one bf16.
template <bool DUAL, int W>
__global__ __launch_bounds__(W* kWave) void grouped_gemm_mx_kernel(GemmArgs a) {
  grouped_gemm_body<W, DUAL, kMx8>(a);
}

// The MXFP8 gate/up reduction: sums the S partials of gate and up for 4
// consecutive columns of a row per thread (16-byte loads, consecutive lanes on
// consecutive columns), applies SiLU(gate) * up as the unsplit epilogue does,
// and quantises each 32-column block (the 8 lanes of an aligned lane group:
// block max by three shuffles, the group's first lane writes the scale code).
// N % 32 == 0 keeps every group inside one block and the item count a
// multiple of 8, so a group is wholly in range or wholly out. Does nothing
// when the GEMM before it split nothing.
__global__ __launch_bounds__(256) void split_reduce_mx_kernel(const float* __restrict__ part,
                                                              const int32_t* __restrict__ plan, int N, int M_cap,
                                                              uint8_t* __restrict__ C8, uint32_t* __restrict__ Cs) {
  const int S = plan[0];
  if (S <= 1) {
    // tail tiles of an unsplit launch; a tile's column count is a multiple
    // of 32, so the 8 lanes of a block share the tile and the row
    const int St = plan[2];
    if (St <= 1) return;
    const size_t items = (size_t)plan[3] * 256 * (plan[4] / 4);
    for (size_t it = (size_t)blockIdx.x * 256 + threadIdx.x; it < items; it += (size_t)gridDim.x * 256) {
      TailItem t;
      if (!tail_item(part, plan, 2, it, t)) continue;
      const float4 g = sum_splits(t.p, t.tsz, St), u = sum_splits(t.p + St * t.tsz, t.tsz, St);
      mx_quant_store4(silu_mul_fast(g.x, u.x), silu_mul_fast(g.y, u.y), silu_mul_fast(g.z, u.z),
                      silu_mul_fast(g.w, u.w), t.row, t.col, N, M_cap, C8, Cs);
    }
    return;
  }
  const int R = plan[1];
  const int n4 = N / 4;
  const size_t items = (size_t)R * n4, sstride = (size_t)R * N, bstride = (size_t)S * R * N;
  for (size_t it = (size_t)blockIdx.x * 256 + threadIdx.x; it < items; it += (size_t)gridDim.x * 256) {
    const int j = (int)(it / n4), c = (int)(it % n4) * 4;
    const float* p = part + (size_t)j * N + c;
    float4 g = *reinterpret_cast<const float4*>(p);
    float4 u = *reinterpret_cast<const float4*>(p + bstride);
    for (int sp = 1; sp < S; ++sp) {
      const float4 a = *reinterpret_cast<const float4*>(p + sp * sstride);
      const float4 b = *reinterpret_cast<const float4*>(p + bstride + sp * sstride);
      g.x += a.x, g.y += a.y, g.z += a.z, g.w += a.w;
      u.x += b.x, u.y += b.y, u.z += b.z, u.w += b.w;
    }
    mx_quant_store4(silu_mul_fast(g.x, u.x), silu_mul_fast(g.y, u.y), silu_mul_fast(g.z, u.z),
                    silu_mul_fast(g.w, u.w), plan[kPlanHead + j], c, N, M_cap, C8, Cs);
  }
}

// ---------------------------------------------------------------------------
// fp32 expert FFN (small layers, a parity configuration): plain VALU dot
// products, a block per row and 32 columns, 8 lanes per column.
//
// A launch is a handful of latencies: the row's expert, one round of loads,
// the sums. With a thread per column, every lane read a weight row of its own
// 16 bytes at a time (64 lines a load, each fetched again for its next piece)
// after a serial scan of the offsets. Here the 8 lanes of a column read whole
// 128-byte lines, lane q taking pieces q, q + 8, ... of the row in ascending
// order, and add up their 8 sums in a tree; a wave looks its row up in 64
// experts at a time. Blocks of neighbouring rows run together and share their
// expert's weights. 128 rows over 8 experts, H = 128, I = 256, us: gate/up
// 13.4 -> 4.9, down 11.7 -> 3.6; error of the outputs against 64 bits 4.4e-7 ->
// 1.9e-7 (shorter chains of sums).
// ---------------------------------------------------------------------------
constexpr int kF32Lanes = 8;             // lanes per column
constexpr int kF32Cols = 256 / kF32Lanes;  // columns per block
constexpr int kF32Blocks = 8192, kF32Rows = 1024;  // blocks of a launch and rows at a time, at least (see launch_ffn)

// The expert whose range holds `row` (the same in every lane), -1 if there is
// none, -2 if none holds any row from `row` on.
__device__ __forceinline__ int find_slot(const int32_t* offsets, int E, int M_cap, int row) {
  uint64_t later = 0;
  for (int e0 = 0; e0 < E; e0 += kWave) {
    const int e = min(e0 + (int)(threadIdx.x & 63), E - 1);
    const int o0 = min(max(offsets[e], 0), M_cap);
    const int o1 = min(max(offsets[e + 1], o0), M_cap);
    const uint64_t in = __ballot(row >= o0 && row < o1);
    if (in != 0) return e0 + __ffsll((unsigned long long)in) - 1;
    later |= __ballot(row < o0 && o0 < o1);
  }
  return later != 0 ? -1 : -2;
}

// Sum over the 8 lanes of a column, in each of them: lanes l ^ 1, l ^ 2, then
// the mirrored lane, which holds the other four's sum.
template <int CTRL>
__device__ __forceinline__ float add_dpp(float v) {
  const int i = __builtin_bit_cast(int, v);
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, CTRL, 0xf, 0xf, false));
}
__device__ __forceinline__ float sum_column(float v) {
  static_assert(kF32Lanes == 8, "three exchanges");
  return add_dpp<0x141>(add_dpp<0x4E>(add_dpp<0xB1>(v)));  // quad_perm 1,0,3,2; 2,3,0,1; row_half_mirror
}

__device__ __forceinline__ void fma4(float4 a, float4 b, float& s) {
  s = __builtin_fmaf(a.x, b.x, s);
  s = __builtin_fmaf(a.y, b.y, s);
  s = __builtin_fmaf(a.z, b.z, s);
  s = __builtin_fmaf(a.w, b.w, s);
}

// 16-byte loads: H, I and ldw are multiples of 4, rows 16-byte aligned.
__global__ __launch_bounds__(256) void gateup_f32_kernel(const float* __restrict__ X, const float* __restrict__ Wg,
                                                         const float* __restrict__ Wu,
                                                         const int32_t* __restrict__ offsets, int E, int M_cap,
                                                         int H, int I, int ldw, float* __restrict__ h) {
  const int q = threadIdx.x % kF32Lanes;
  for (int row = blockIdx.x; row < M_cap; row += gridDim.x) {
    const int e = find_slot(offsets, E, M_cap, row);
    if (e == -2) return;
    if (e < 0) continue;
    const float4* x = reinterpret_cast<const float4*>(X + (size_t)row * H);
    for (int i0 = blockIdx.y * kF32Cols; i0 < I; i0 += gridDim.y * kF32Cols) {
      const int i = i0 + threadIdx.x / kF32Lanes;
      const size_t w0 = ((size_t)e * I + min(i, I - 1)) * ldw;  // columns past the last one read it again
      const float4* wg = reinterpret_cast<const float4*>(Wg + w0);
      const float4* wu = reinterpret_cast<const float4*>(Wu + w0);
      float g = 0.0f, u = 0.0f;
#pragma unroll 4
      for (int c = q; c < H / 4; c += kF32Lanes) {
        const float4 xv = x[c], gv = wg[c], uv = wu[c];
        fma4(xv, gv, g);
        fma4(xv, uv, u);
      }
      g = sum_column(g);
      u = sum_column(u);
      if (q == 0 && i < I) h[(size_t)row * I + i] = silu_mul(g, u);
    }
  }
}

__global__ __launch_bounds__(256) void down_f32_kernel(const float* __restrict__ h, const float* __restrict__ Wd,
                                                       const int32_t* __restrict__ offsets, int E, int M_cap, int H,
                                                       int I, int ldw, float* __restrict__ y) {
  const int q = threadIdx.x % kF32Lanes;
  for (int row = blockIdx.x; row < M_cap; row += gridDim.x) {
    const int e = find_slot(offsets, E, M_cap, row);
    if (e == -2) return;
    if (e < 0) continue;
    const float4* hr = reinterpret_cast<const float4*>(h + (size_t)row * I);
    for (int c0 = blockIdx.y * kF32Cols; c0 < H; c0 += gridDim.y * kF32Cols) {
      const int c = c0 + threadIdx.x / kF32Lanes;
      const float4* wd = reinterpret_cast<const float4*>(Wd + ((size_t)e * H + min(c, H - 1)) * ldw);
      float s = 0.0f;
#pragma unroll 8
      for (int i = q; i < I / 4; i += kF32Lanes) fma4(hr[i], wd[i], s);
      s = sum_column(s);
      if (q == 0 && c < H) y[(size_t)row * H + c] = s;
    }
  }
}

// Zeroes the work counters at the start of the scratch of the entry point
// that allocates nothing, at its first use on a device (a kernel, not a
// memset, so that a first call under graph capture records no memset).
__global__ void clear_counters_kernel(int32_t* q, int n) {
  for (int i = (int)threadIdx.x; i < n; i += (int)blockDim.x) q[i] = 0;
}

__global__ void set_offsets_kernel(int32_t* offsets, int m) {
  if (threadIdx.x == 0) {
    offsets[0] = 0;
    offsets[1] = m;
  }
}

// ---------------------------------------------------------------------------
// Launchers
// ---------------------------------------------------------------------------
// bf16 workspace: counters (kCntBytes at offset 0, the same place whatever
// the sizes, so a buffer can serve calls of any size) | h [M_cap, I] |
// split-K plan | fp32 partials (split-K, tail split or the decode
// schedule's slots). The counters must be zero before the first call on a
// workspace; every call leaves them zero. A split
// launch has R <= M_cap partial rows for offsets that are a valid scan (and
// R <= 64 E_local when every expert is small), and S <= 8. The kernel splits
// only when R fits the plan's row map and its partials fit in part_cap.
struct FfnWs {
  size_t h, plan, part;  // byte offsets
  long long part_cap;    // floats
  int plan_rows;         // rows of the plan's row map
  bool sk_ok;            // the partial region holds the decode schedule's slots
  size_t bytes;
};

// fp32 partials either split-K (S <= kMaxSplit slices of every row of both
// GEMMs) or the tail split (at most 256 split tiles of 256 x 256 floats, and
// at most kMaxSplit per tile) may need, within kPartCapFloats.
static long long part_cap_floats(int M_cap, int E_local, int H, int I) {
  const long long split_k = (long long)kMaxSplit * M_cap * std::max(2LL * I, (long long)H);
  const long long tiles = ((long long)(M_cap + kSmallM - 1) / kSmallM + E_local) * (std::max(I, H) / 128);
  const long long tail = std::min(256LL, (long long)kMaxSplit * tiles) * 256 * 256;
  return std::min(std::max(split_k, tail), kPartCapFloats);
}

// Layout of an FFN workspace of at most `cap` bytes (SIZE_MAX: as large as
// the call can use). A smaller capacity shrinks only the partial region:
// fewer tiles can then split, and below the slots' size the decode schedule
// is off. The fixed part (counters, h, plan) must fit: see ffn_ws_fixed.
static FfnWs ffn_ws_layout(int M_cap, int E_local, int H, int I, bool bf16, size_t cap = SIZE_MAX) {
  FfnWs w{};
  const size_t h = round256((size_t)M_cap * I * (bf16 ? 2 : 4));
  w.h = 0;
  if (!bf16) {
    w.bytes = h + 256;
    return w;
  }
  w.h = kCntBytes;
  w.plan_rows = std::max(M_cap, kSmallM * E_local);
  w.plan = w.h + h;
  w.part = w.plan + round256((size_t)(kPlanHead + (size_t)w.plan_rows) * 4);
  const long long full = std::max(part_cap_floats(M_cap, E_local, H, I), sk_slot_floats());
  size_t part_bytes = round256((size_t)full * 4);
  if (cap != SIZE_MAX) part_bytes = std::min(part_bytes, cap > w.part ? ((cap - w.part) & ~(size_t)255) : 0);
  w.part_cap = std::min(part_cap_floats(M_cap, E_local, H, I), (long long)(part_bytes / 4));
  w.sk_ok = (long long)(part_bytes / 4) >= sk_slot_floats();
  w.bytes = w.part + part_bytes;
  return w;
}

size_t ffn_ws_fixed(int M_cap, int E_local, int H, int I, bool bf16) {
  const FfnWs w = ffn_ws_layout(M_cap, E_local, H, I, bf16, 0);
  return bf16 ? w.part : w.bytes;
}

size_t ffn_ws_bytes(int M_cap, int E_local, int H, int I, bool bf16) {
  return ffn_ws_layout(M_cap, E_local, H, I, bf16).bytes;
}

int device_cu_count() {
  static int cached[64] = {0};
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
  if (cached[dev] == 0) {
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
    cached[dev] = n;
  }
  return cached[dev];
}

// XCD check. The decode schedule keeps partial sums in an XCD's L2 only if
// the blocks that share them run on one XCD, i.e. if workgroup b of a launch
// runs on XCD b % 8 (the hardware deals workgroups to the XCDs round robin).
// This kernel checks that once per device: block b compares the XCC_ID
// hardware register with b % 8; the last block to finish publishes the
// result in st[0] (1: every block matched, 2: some did not; 0 until then).
// st[1] counts mismatches, st[2] finished blocks. It has the GEMMs' block
// size and holds a comparable share of LDS, so blocks are placed as theirs.
static __device__ int32_t xcd_check[4];
__global__ __launch_bounds__(kMaxWaves* kWave) void xcd_probe_kernel(int32_t* st) {
  __shared__ int32_t s_pad[32768];
  int x;
  asm volatile("s_getreg_b32 %0, hwreg(HW_REG_XCC_ID, 0, 4)" : "=s"(x));
  s_pad[threadIdx.x * 64] = x;
  __syncthreads();
  if (threadIdx.x == 0) {
    if (s_pad[0] != (int)(blockIdx.x & 7)) atomicAdd(st + 1, 1);
    __threadfence();
    if (atomicAdd(st + 2, 1) == (int)gridDim.x - 1) {
      __threadfence();
      const int bad = __hip_atomic_load(st + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      __hip_atomic_store(st, bad == 0 ? 1 : 2, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
}

// The XCD check's result on the current device for a launch on stream s,
// or nullptr (kernels then keep partial sums at the point of coherence; the
// results are the same). The check is launched on stream s by the first call
// on the device that is not under graph capture. Its result goes to launches
// on that stream (ordered after it) and, once the check has completed, to
// launches on any stream, so that no launch runs while the result changes.
const int32_t* xcd_state(hipStream_t s) {
  struct Dev {
    int32_t* ptr;
    hipEvent_t done;
    hipStream_t stream;
    bool launched, ready;
  };
  static std::mutex mu;
  static Dev devs[64] = {};
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return nullptr;
  std::lock_guard<std::mutex> lock(mu);
  Dev& d = devs[dev];
  if (d.ptr == nullptr) {
    void* p = nullptr;
    if (hipGetSymbolAddress(&p, HIP_SYMBOL(xcd_check)) != hipSuccess || p == nullptr) {
      (void)hipGetLastError();
      return nullptr;
    }
    d.ptr = static_cast<int32_t*>(p);
  }
  // no launch, event record or event query under graph capture (they could
  // end it); the result is then passed on only if it is known
  hipStreamCaptureStatus cs = hipStreamCaptureStatusActive;
  const bool capturing = hipStreamIsCapturing(s, &cs) != hipSuccess || cs != hipStreamCaptureStatusNone;
  if (capturing) (void)hipGetLastError();
  if (!d.launched) {
    if (capturing) return nullptr;
    if (d.done == nullptr && hipEventCreateWithFlags(&d.done, hipEventDisableTiming) != hipSuccess) {
      (void)hipGetLastError();
      d.done = nullptr;
      return nullptr;
    }
    xcd_probe_kernel<<<kMaxBlocks, kMaxWaves * kWave, 0, s>>>(d.ptr);
    if (hipGetLastError() != hipSuccess || hipEventRecord(d.done, s) != hipSuccess) {
      (void)hipGetLastError();
      return nullptr;
    }
    d.launched = true;
    d.stream = s;
  }
  if (!d.ready && !capturing) {
    const hipError_t q = hipEventQuery(d.done);
    if (q == hipSuccess)
      d.ready = true;
    else if (q != hipErrorNotReady)
      (void)hipGetLastError();
  }
  return d.ready || s == d.stream ? d.ptr : nullptr;
}

hipError_t launch_ffn(const void* x_perm, const void* w_gate, const void* w_up, const void* w_down,
                      const int32_t* offsets, int E_local, int H, int I, int ld_gu, int ld_dn, int M_cap, bool bf16,
                      void* y_perm, void* ws, hipStream_t s, const int32_t* a_src, int a_div, int a_T,
                      size_t ws_cap, int rows) {
  if (E_local == 0 || M_cap == 0) return hipSuccess;
  const FfnWs L = ffn_ws_layout(M_cap, E_local, H, I, bf16, ws_cap);
  char* wsb = static_cast<char*>(ws);
  void* h = wsb + L.h;
  if (!bf16) {
    // Enough blocks for every CU several times over, and the rows of an expert
    // side by side (they share its weights in the L2: with 93 rows at a time
    // 1000 rows over 16 experts, H = 1024, I = 2816, took 2787 us, with all of
    // them 2006); the kernels loop over the rest. M_cap counts rows of remote
    // experts too: with a block per row of it, 128 local rows of 65536 (H = 128,
    // I = 256) took 256 us, now 12.
    auto grid = [&](int N) {
      const int cols = std::min((N - 1) / kF32Cols + 1, 65535);
      return dim3((unsigned)std::min(M_cap, std::max(kF32Blocks / cols, kF32Rows)), (unsigned)cols);
    };
    gateup_f32_kernel<<<grid(I), 256, 0, s>>>(
        static_cast<const float*>(x_perm), static_cast<const float*>(w_gate), static_cast<const float*>(w_up),
        offsets, E_local, M_cap, H, I, ld_gu, static_cast<float*>(h));
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    down_f32_kernel<<<grid(H), 256, 0, s>>>(static_cast<const float*>(h), static_cast<const float*>(w_down), offsets,
                                            E_local, M_cap, H, I, ld_dn, static_cast<float*>(y_perm));
    return hipGetLastError();
  }
  const int cus = device_cu_count();
  // Upper bound on unsplit tiles: every expert could need one partial tile
  // plus ceil(rows / 64) full ones. The grid is a multiple of 8 (one share
  // per XCD). A split launch has S times the tiles of a launch with fewer
  // tiles than blocks, so the grid covers at least 8 of those.
  auto grid_for = [&](int N) {
    const long long ub = ((long long)(M_cap + kSmallM - 1) / kSmallM + E_local) * (N / 128) * kMaxSplit;
    long long g = std::min(cus, kMaxBlocks);  // one block per CU
    if (ub < g) g = ub;
    if (g >= 8) g &= ~7LL;
    return (unsigned)(g < 1 ? 1 : g);
  };
  float* part = reinterpret_cast<float*>(wsb + L.part);
  int32_t* plan = reinterpret_cast<int32_t*>(wsb + L.plan);
  int32_t* cnt = reinterpret_cast<int32_t*>(wsb);
  // reduce grid: one float4 column group per thread, grid-stride over 4
  // blocks per CU (a split launch has up to max(M_cap, 64 E_local) rows of
  // N columns to finish, a tail split up to G / 2 tiles of 256 x 256)
  auto reduce_grid = [&](int) { return (unsigned)(4 * cus); };
  // The GEMMs take the decode schedule when no expert has more than
  // kSkHostRows rows (or, tile-starved, kSkRows), and finish its split tiles
  // inside their launches. When no expert can have more than kSkHostRows (a
  // token contributes at most one row to an expert, so with the row gather
  // the bound is min(T, M_cap)), the reduction launches are skipped: the
  // call is two launches.
  const int row_bound = a_src != nullptr ? std::min(a_T, M_cap) : M_cap;
  const bool sk = L.sk_ok && row_bound <= kSkHostRows;
  GemmArgs g1{static_cast<const bf16_t*>(x_perm), static_cast<const bf16_t*>(w_gate),
              static_cast<const bf16_t*>(w_up), static_cast<bf16_t*>(h), offsets, E_local, M_cap, I, H,
              part, L.part_cap, plan, L.plan_rows};
  g1.queue = cnt + kQueueGU;
  g1.done = cnt + kDoneGU;
  g1.a_src = a_src;
  g1.a_div = a_div;
  g1.a_T = a_T;
  g1.ldb = ld_gu;
  g1.sk = L.sk_ok ? 1 : 0;
  g1.no_reduce = sk ? 1 : 0;
  g1.sk_rows = kSkRows;
  g1.skpart = part;
  g1.tcnt = cnt + kTcntGU;
  g1.xcd_state = L.sk_ok ? xcd_state(s) : nullptr;
  hipError_t e = launch_waves(sk ? Waves::k8 : waves_for(true, M_cap, E_local, I, H, rows), g1, grid_for(I), s,
                   grouped_gemm_bf16_kernel<true, 4>, grouped_gemm_bf16_kernel<true, 8>);
  if (e != hipSuccess) return e;
  // A GEMM can split only if its K range holds two splits of kMinSplitChunks.
  const bool split_gu = H / kBK >= 2 * kMinSplitChunks, split_dn = I / kBK >= 2 * kMinSplitChunks;
  if (split_gu && !sk) {
    split_reduce_kernel<true><<<reduce_grid(I), 256, 0, s>>>(part, plan, I, static_cast<bf16_t*>(h));
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  GemmArgs g2{static_cast<const bf16_t*>(h), static_cast<const bf16_t*>(w_down), nullptr,
              static_cast<bf16_t*>(y_perm), offsets, E_local, M_cap, H, I, part, L.part_cap, plan, L.plan_rows};
  g2.queue = cnt + kQueueDN;
  g2.done = cnt + kDoneDN;
  g2.ldb = ld_dn;
  g2.sk = g1.sk;
  g2.no_reduce = g1.no_reduce;
  g2.sk_rows = kSkRows;
  g2.skpart = part;
  g2.tcnt = cnt + kTcntDN;
  g2.xcd_state = g1.xcd_state;
  e = launch_waves(sk ? Waves::k8 : waves_for(false, M_cap, E_local, H, I, rows), g2, grid_for(H), s,
                   grouped_gemm_bf16_kernel<false, 4>, grouped_gemm_bf16_kernel<false, 8>);
  if (e != hipSuccess) return e;
  if (split_dn && !sk)
    split_reduce_kernel<false><<<reduce_grid(H), 256, 0, s>>>(part, plan, H, static_cast<bf16_t*>(y_perm));
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// MXFP8 expert FFN: gate/up (MXFP8 in, MXFP8 h out), then down (bf16 out)
// ---------------------------------------------------------------------------
// MXFP8 FFN workspace: counters (kCntBytes, zero before first use, as for
// bf16) | h codes [M_cap, I] | h scale dwords [I/128][M_cap] | split-K plan |
// fp32 partials (split-K, or the decode schedule's slots).
struct FfnMxWs {
  size_t hq, hs, plan, part;  // byte offsets
  long long part_cap;
  int plan_rows;
  size_t bytes;
};

static FfnMxWs ffn_mx_ws_layout(int M_cap, int E_local, int H, int I) {
  FfnMxWs w{};
  w.hq = kCntBytes;
  w.hs = w.hq + round256((size_t)M_cap * I);
  w.plan = w.hs + round256((size_t)(I / kMxChunk) * M_cap * 4);
  // sized for split-K only, not for the tail split as the bf16 layout is:
  // with room for it, the MXFP8 decode FFN (Mixtral-shaped, T = 32) took the
  // tail split over S = 2 and measured 3 % slower
  const long long need = (long long)kMaxSplit * M_cap * std::max(2LL * I, (long long)H);
  w.part_cap = std::min(need, kPartCapFloats);
  w.plan_rows = std::max(M_cap, kSmallM * E_local);
  w.part = w.plan + round256((size_t)(kPlanHead + (size_t)w.plan_rows) * 4);
  w.bytes = w.part + round256((size_t)std::max(w.part_cap, sk_slot_floats()) * 4);
  return w;
}

size_t ffn_mx_ws_bytes(int M_cap, int E_local, int H, int I) {
  return ffn_mx_ws_layout(M_cap, E_local, H, I).bytes;
}

static hipError_t gateup_mx(const uint8_t* xq, const uint32_t* xs, const uint8_t* wgq, const uint32_t* wgs,
                            const uint8_t* wuq, const uint32_t* wus, const int32_t* offsets, int E_local, int H,
                            int I, int ldw, int M_cap, uint8_t* hq, uint32_t* hs, const MxSplit& sp,
                            hipStream_t s, int rows = 0) {
  GemmArgs g{};
  g.A = reinterpret_cast<const bf16_t*>(xq);
  g.B0 = reinterpret_cast<const bf16_t*>(wgq);
  g.B1 = reinterpret_cast<const bf16_t*>(wuq);
  g.C = reinterpret_cast<bf16_t*>(hq);
  g.offsets = offsets;
  g.E_local = E_local;
  g.M_cap = M_cap;
  g.N = I;
  g.K = H;
  g.ldb = ldw;
  mx_split_args(g, sp);
  g.As = xs;
  g.Bs0 = wgs;
  g.Bs1 = wus;
  g.Cs = hs;
  const bool split = sp.plan != nullptr && H / kMxChunk >= 2 * kMinSplitChunks;
  hipError_t e = launch_waves(waves_for(true, M_cap, E_local, I, H, rows), g, mx_grid(M_cap, E_local, I, split || g.sk),
                              s, grouped_gemm_mx_kernel<true, 4>, grouped_gemm_mx_kernel<true, 8>);
  if (e != hipSuccess || !split || sp.no_reduce) return e;
  split_reduce_mx_kernel<<<mx_reduce_grid(sp.plan_rows, I / 4), 256, 0, s>>>(sp.part, sp.plan, I, M_cap,
                                                                                     hq, hs);
  return hipGetLastError();
}

static hipError_t gemm_mx(const uint8_t* aq, const uint32_t* as, const uint8_t* bq, const uint32_t* bs,
                          const int32_t* offsets, int E_local, int N, int K, int ldb, int M_cap, void* c,
                          const MxSplit& sp, hipStream_t s, int rows = 0) {
  GemmArgs g{};
  g.A = reinterpret_cast<const bf16_t*>(aq);
  g.B0 = reinterpret_cast<const bf16_t*>(bq);
  g.C = static_cast<bf16_t*>(c);
  g.offsets = offsets;
  g.E_local = E_local;
  g.M_cap = M_cap;
  g.N = N;
  g.K = K;
  g.ldb = ldb;
  mx_split_args(g, sp);
  g.As = as;
  g.Bs0 = bs;
  const bool split = sp.plan != nullptr && K / kMxChunk >= 2 * kMinSplitChunks;
  hipError_t e = launch_waves(waves_for(false, M_cap, E_local, N, K, rows), g,
                              mx_grid(M_cap, E_local, N, split || g.sk), s, grouped_gemm_mx_kernel<false, 4>,
                              grouped_gemm_mx_kernel<false, 8>);
  if (e != hipSuccess || !split || sp.no_reduce) return e;
  split_reduce_kernel<false><<<mx_reduce_grid(sp.plan_rows, N / 4), 256, 0, s>>>(sp.part, sp.plan, N,
                                                                                  static_cast<bf16_t*>(c));
  return hipGetLastError();
}

hipError_t launch_gateup_mx(const uint8_t* xq, const uint32_t* xs, const uint8_t* wgq, const uint32_t* wgs,
                            const uint8_t* wuq, const uint32_t* wus, const int32_t* offsets, int E_local, int H,
                            int I, int ldw, int M_cap, uint8_t* hq, uint32_t* hs, hipStream_t s) {
  if (E_local == 0 || M_cap == 0) return hipSuccess;
  return gateup_mx(xq, xs, wgq, wgs, wuq, wus, offsets, E_local, H, I, ldw, M_cap, hq, hs, MxSplit{}, s);
}

hipError_t launch_gemm_mx(const uint8_t* aq, const uint32_t* as, const uint8_t* bq, const uint32_t* bs,
                          const int32_t* offsets, int E_local, int N, int K, int ldb, int M_cap, void* c,
                          hipStream_t s) {
  if (E_local == 0 || M_cap == 0) return hipSuccess;
  return gemm_mx(aq, as, bq, bs, offsets, E_local, N, K, ldb, M_cap, c, MxSplit{}, s);
}

hipError_t launch_ffn_mx(const uint8_t* xq, const uint32_t* xs, const uint8_t* wgq, const uint32_t* wgs,
                         const uint8_t* wuq, const uint32_t* wus, const uint8_t* wdq, const uint32_t* wds,
                         const int32_t* offsets, int E_local, int H, int I, int ld_gu, int ld_dn, int M_cap,
                         void* y_perm, void* ws, hipStream_t s, int rows) {
  if (E_local == 0 || M_cap == 0) return hipSuccess;
  const FfnMxWs L = ffn_mx_ws_layout(M_cap, E_local, H, I);
  char* w = static_cast<char*>(ws);
  uint8_t* hq = reinterpret_cast<uint8_t*>(w + L.hq);
  uint32_t* hs = reinterpret_cast<uint32_t*>(w + L.hs);
  int32_t* cnt = reinterpret_cast<int32_t*>(w);
  // as in launch_ffn: the decode schedule finishes its split tiles inside the
  // GEMM launches; when no expert can exceed kSkHostRows rows no reduction
  // follows
  const bool no_reduce = M_cap <= kSkHostRows;
  const MxSplit sp1{reinterpret_cast<float*>(w + L.part), L.part_cap, reinterpret_cast<int32_t*>(w + L.plan),
                    L.plan_rows, cnt + kQueueGU, cnt + kDoneGU, cnt + kTcntGU, no_reduce, xcd_state(s)};
  hipError_t e = gateup_mx(xq, xs, wgq, wgs, wuq, wus, offsets, E_local, H, I, ld_gu, M_cap, hq, hs, sp1, s,
                          rows);
  if (e != hipSuccess) return e;
  const MxSplit sp2{sp1.part, sp1.part_cap, sp1.plan, sp1.plan_rows, cnt + kQueueDN, cnt + kDoneDN, cnt + kTcntDN,
                    no_reduce, sp1.xcd};
  return gemm_mx(hq, hs, wdq, wds, offsets, E_local, H, I, ld_dn, M_cap, y_perm, sp2, s, rows);
}

// ---------------------------------------------------------------------------
// Router logits by K ranges (the router GEMM z = x W_r^T for many tokens and
// E = 128 or 256 experts): block (t, s) sums x[256 t, +256) W_r^T over the K
// chunks [s nK / S, (s + 1) nK / S) with the expert FFN's 256-row tile and
// writes the fp32 sums to part[s][row][0, E); gate_topk_reduce_kernel adds the
// S slices in split order. A CU then loads 256 token rows and the E router
// rows of one K range, where a router block that finishes its tokens' top-k
// itself loads all E router rows for every 64 tokens.
// ---------------------------------------------------------------------------
template <int BN>
__global__ __launch_bounds__(512) void router_logits_split_kernel(GemmArgs a, int S, float* __restrict__ part) {
  __shared__ __align__(16) bf16_t smem[Stages<256, BN, false, 8>::BYTES / 2];
  const int T = a.M_cap;
  const int m0 = (int)blockIdx.x * 256;
  const int m_end = min(m0 + 256, T);
  const int nK = a.K / kBK, sp = (int)blockIdx.y;
  const int kc0 = sp * nK / S, kc1 = (sp + 1) * nK / S;
  float* pbase = part + ((size_t)sp * T + m0) * BN;
  gemm_tile<8, 256, BN, 4, false, true, false, 64>(a, smem, 0, m0, m_end, 0, kc0, kc1, pbase, 0, BN, 0);
}

hipError_t launch_router_logits_split(const void* x, const void* wr, int T, int H, int E, int S, float* part,
                                      hipStream_t s) {
  if (T < 1 || S < 1 || S > 8 || H % kBK != 0 || H / kBK < S) return hipErrorInvalidValue;
  GemmArgs g{};
  g.A = static_cast<const bf16_t*>(x);
  g.B0 = static_cast<const bf16_t*>(wr);
  g.E_local = 1;
  g.M_cap = T;
  g.N = E;
  g.K = H;
  g.ldb = H;
  const dim3 grid((unsigned)((T + 255) / 256), (unsigned)S);
  if (E == 256)
    router_logits_split_kernel<256><<<grid, 512, 0, s>>>(g, S, part);
  else if (E == 128)
    router_logits_split_kernel<128><<<grid, 512, 0, s>>>(g, S, part);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Scratch of the FFN entry point that allocates nothing
// (moe_grouped_swiglu_ffn_noalloc): the workspace of its calls, one copy per
// GPU in the code object's device memory, held until the process ends. In
// host code `scratch` only names the symbol; its address on a device comes
// from hipGetSymbolAddress with that device current, and only that address
// is passed to kernels.
// ---------------------------------------------------------------------------
static __device__ __align__(256) unsigned char scratch[kScratchBytes];

hipError_t ffn_scratch(void** out, hipStream_t s) {
  static std::mutex mu;
  static void* ptrs[64] = {nullptr};
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= 64) return hipErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(mu);
  if (ptrs[dev] == nullptr) {
    void* p = nullptr;
    e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
    if (e != hipSuccess) return e;
    if (p == nullptr) return hipErrorInvalidSymbol;
    // the counters must start at zero (every call leaves them zero); a
    // kernel rather than a memset, so that a first call under graph capture
    // records no memset node
    clear_counters_kernel<<<1, 1024, 0, s>>>(static_cast<int32_t*>(p), (int)(kCntBytes / 4));
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    ptrs[dev] = p;
  }
  *out = ptrs[dev];
  return hipSuccess;
}

hipError_t launch_set_offsets(int32_t* offsets, int m, hipStream_t s) {
  set_offsets_kernel<<<1, 64, 0, s>>>(offsets, m);
  return hipGetLastError();
}

}  // namespace moe
