// Gradient of the router's product z = x W^T + b (gfx950): dx = dz W, dW = dz^T x,
// db = sum_t dz.
//
// dz is fp32, x and W bf16, and the MFMA takes bf16 pairs: dz is cut into bf16
// terms, each multiplied with the exact other operand and summed in fp32. For dW,
// fp32 like the sums, three terms hold all 24 bits of an element; for dx, rounded
// to bf16 (2^-8 of its value), two rounded to nearest are enough: they are off by at
// most 2^-17 of an element, in either direction. (Cut off, as the three are, two would
// lose up to 2^-15, always towards zero, which shows where dx is small beside its
// terms: rows of dz sum to nearly nothing, and the rows of W may have much in common.)
// Both reductions run along a dimension that is a row index of the bf16 operand
// (tokens of x, experts of W), so its fragments are read from LDS with the
// transposing read.
#include <algorithm>
#include <type_traits>

#include "common.hpp"
#include "grouped_gemm.hpp"
#include "launch.hpp"

namespace moe {

typedef short s16x4_t __attribute__((ext_vector_type(4)));

// Fragment of 32 columns x 16 rows of a bf16 tile in LDS with 256-byte rows, for
// an operand whose reduction dimension is the tile's row: lane (c = lane % 32, h =
// lane / 32) gets rows k0 + 8 h + (0..7) of column c0 + c. A transposing read takes
// 16 lanes x 8 bytes as 4 rows x 16 columns and hands lane i column i; the 16-byte
// pieces of a row are swizzled by 64 bytes per row, so that the four rows lie in
// different banks. `at` is the lane's byte offset (tr_offset), in which k0 and c0
// are added as whole rows and 64-byte groups.
__device__ __forceinline__ int tr_swizzle(int row, int piece) { return piece ^ ((row & 3) << 2); }
__device__ __forceinline__ uint32_t tr_row(int lane) { return (uint32_t)(8 * (lane >> 5) + ((lane & 15) >> 2)); }
__device__ __forceinline__ bf16x8_t tr_frag(const char* tile, int lane, int k0, int c0) {
  const int row = (int)tr_row(lane), colb = c0 * 2 + 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
  const uint32_t off = (uint32_t)((k0 + row) * 256 + tr_swizzle(row, colb >> 4) * 16 + (colb & 15));
  typedef __attribute__((address_space(3))) s16x4_t* lds4;
  const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(tile)) + off;
  const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds4>(base));
  const s16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds4>(base + 4 * 256));
  struct {
    s16x4_t lo, hi;
  } v = {a, b};
  return __builtin_bit_cast(bf16x8_t, v);
}

// Eight fp32 values as three bf16 fragments, f = sum of frag[n]: each takes the upper
// 16 bits of what is left (the differences are exact).
__device__ __forceinline__ void split8(float (&f)[8], bf16x8_t (&frag)[3]) {
#pragma unroll
  for (int n = 0; n < 3; ++n) {
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      w[q] = __builtin_amdgcn_perm(__float_as_uint(f[2 * q + 1]), __float_as_uint(f[2 * q]), 0x07060302u);
    frag[n] = as_bf16x8(make_uint4(w[0], w[1], w[2], w[3]));
    if (n + 1 < 3)
#pragma unroll
      for (int q = 0; q < 8; ++q) f[q] -= __uint_as_float(__float_as_uint(f[q]) & 0xffff0000u);
  }
}

// Eight fp32 values as two bf16 fragments: f rounded to nearest, and what that left
// (exact in fp32), rounded to nearest. The first stays within bf16's finite range, so
// that a value which would round up to infinity does not.
__device__ __forceinline__ void split8_nearest(const float (&f)[8], bf16x8_t (&frag)[2]) {
  constexpr float kMaxBf16 = 0x1.fep127f;
  uint32_t hi[4], lo[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    hi[q] = pack_bf16x2(__builtin_amdgcn_fmed3f(f[2 * q], -kMaxBf16, kMaxBf16),
                        __builtin_amdgcn_fmed3f(f[2 * q + 1], -kMaxBf16, kMaxBf16));
    lo[q] = pack_bf16x2(f[2 * q] - __uint_as_float(hi[q] << 16),
                        f[2 * q + 1] - __uint_as_float(hi[q] & 0xffff0000u));
  }
  frag[0] = as_bf16x8(make_uint4(hi[0], hi[1], hi[2], hi[3]));
  frag[1] = as_bf16x8(make_uint4(lo[0], lo[1], lo[2], lo[3]));
}

// ---------------------------------------------------------------------------
// dW and db: a block sums E x 128 columns of x over its range of tokens, 32 at a
// time: the chunk's dz rows (fp32) and x rows (128 columns) go to LDS by direct
// loads, NS stages deep. A wave holds 32 experts by all 128 columns (EP = 256), so
// every dz value is cut into its terms once, by the wave that owns its expert, as
// it is read (lanes across experts: a row of LDS is read without conflicts). Two
// waves on a SIMD: one's MFMAs run while the other cuts.
// 16384 tokens, H = 7168, E = 256 take 190-240 us (60 GFLOP, three times that on the
// MFMAs: 0.75-0.95 PFLOP/s): 372 thousand cycles, MFMAs busy in 43 % of them, the rest
// the reads and cuts of dz; at a clock of 2.3 GHz 169 us (launches with pauses between
// them), in a row at what power leaves. Two terms lost bits (relative error 2.5e-6 for
// 2e-7); the 60 GFLOP alone take 390 us at the rate of a large fp32 product.
// Experts past E are computed from other rows' values and not stored. Blocks of one
// token range follow each other by the number of ranges, so that (for 2, 4 or 8 of
// them) an XCD works on one or a few ranges and reads their dz from its L2.
// ---------------------------------------------------------------------------
constexpr int kRgTok = 32;    // tokens of a chunk
constexpr int kRgCols = 128;  // columns of x of a block

struct RouterGradArgs {
  const float* dz;   // [T, E]
  const bf16_t* x;   // [T, H]
  const bf16_t* w;   // [E, H]
  bf16_t* dx;        // [T, H]
  float* dw;         // [S][E][H] partial sums, or dW
  float* db;         // [S][E]
  int T, E, H;
  int S;             // token ranges
};

template <int EP>
struct RgStage {
  static constexpr int DZ = kRgTok * EP * 4;             // bytes of dz
  static constexpr int BYTES = DZ + kRgTok * kRgCols * 2;
  static constexpr int FIT = 150 * 1024 / BYTES;
  static constexpr int NS = FIT > 4 ? 4 : FIT;
};

// VEC: E % 4 == 0, dz rows are whole 16-byte pieces.
template <int EP, bool VEC>
__global__ __launch_bounds__(512) void router_dw_kernel(RouterGradArgs a) {
  using St = RgStage<EP>;
  constexpr int W = 8, WE = EP / 32, WC = W / WE;       // waves along experts, columns
  constexpr int NJ = kRgCols / (32 * WC);               // 32 x 32 blocks of a wave
  constexpr int WCOLS = kRgCols / WC;
  __shared__ __align__(16) bf16_t smem[St::BYTES * St::NS / 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WC, wn = wave % WC, r32 = lane & 31, h = lane >> 5;
  const int E = a.E, H = a.H;
  const int sp = (int)(blockIdx.x % (unsigned)a.S), tile = (int)(blockIdx.x / (unsigned)a.S);
  const int c0 = tile * kRgCols;
  const int chunks = (a.T - 1) / kRgTok + 1;
  const int q0 = uniform_int((int)((long long)sp * chunks / a.S));
  const int q1 = uniform_int((int)((long long)(sp + 1) * chunks / a.S));

  // Direct loads. dz: 1 KB of a stage per instruction, 16 bytes a lane (VEC) or 256
  // bytes, 4 a lane; columns past E read the row's last ones. x: 4 rows of 256
  // bytes; columns past H read the row's last ones. Rows past T read the last.
  constexpr int DL = VEC ? 16 : 4, ND = St::DZ / (64 * DL * W), NX = kRgTok * kRgCols * 2 / (1024 * W);
  constexpr int LOADS = ND + NX;
  static_assert(LOADS * (St::NS - 2) < 64, "loads that a wait counts");
  uint32_t dcol[ND], xcol[NX];
#pragma unroll
  for (int i = 0; i < ND; ++i) dcol[i] = (uint32_t)min(((i * W + wave) * 64 + lane) * DL % (EP * 4), E * 4 - DL);
#pragma unroll
  for (int i = 0; i < NX; ++i)
    xcol[i] = (uint32_t)min(c0 + tr_swizzle((i * W + wave) * 4 + lane / 16, lane % 16) * 8, H - 8) * 2u;
  auto issue = [&](int q, bool live, bf16_t* st, int part) {
    if (part > 0) return;  // all at once
    const int t0 = (live ? q0 + q : q1 - 1) * kRgTok, last = a.T - 1 - t0;
    const void* dz = uniform_ptr(a.dz + (size_t)t0 * E);
    const void* x = uniform_ptr(a.x + (size_t)t0 * H);
    const uint32_t lds = lds_addr(st);
#pragma unroll
    for (int i = 0; i < ND; ++i) {
      const int row = ((i * W + wave) * 64 + lane) * DL / (EP * 4);
      const uint32_t off = (uint32_t)min(row, last) * (uint32_t)(E * 4) + dcol[i];
      if (VEC)
        dma16a(dz, off, lds + (i * W + wave) * 64 * DL);
      else
        dma4a(dz, off, lds + (i * W + wave) * 64 * DL);
    }
#pragma unroll
    for (int i = 0; i < NX; ++i) {
      const int row = (i * W + wave) * 4 + lane / 16;
      dma16a(x, (uint32_t)min(row, last) * (uint32_t)(H * 2) + xcol[i], lds + St::DZ + (i * W + wave) * 1024);
    }
  };

  f32x16_t acc[NJ];
#pragma unroll
  for (int j = 0; j < NJ; ++j) acc[j] = f32x16_t{};
  float db = 0.0f;
  const int e_lane = wm * 32 + r32;  // this lane's expert
  // Raw operands of a 16-token step are read one step ahead, across chunks too
  // (pipeline_xk); a step cuts its dz values and multiplies.
  float f[2][8];
  bf16x8_t xf[2][NJ];
  auto read = [&](const bf16_t* st, int s, int buf) {
    const char* base = reinterpret_cast<const char*>(st);
    const float* dz = reinterpret_cast<const float*>(base);
#pragma unroll
    for (int k = 0; k < 8; ++k) f[buf][k] = dz[(16 * s + 8 * h + k) * EP + e_lane];
#pragma unroll
    for (int j = 0; j < NJ; ++j) xf[buf][j] = tr_frag(base + St::DZ, lane, 16 * s, wn * WCOLS + j * 32);
  };
  int left = a.T - q0 * kRgTok;  // tokens from the present step on
  auto mma = [&](int s) {
    const int buf = s & 1;
    if (left < 16) {
      // past the last token: zeros on both sides, so that they add nothing
#pragma unroll
      for (int k = 0; k < 8; ++k) f[buf][k] = 8 * h + k < left ? f[buf][k] : 0.0f;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        u32x4_t v = __builtin_bit_cast(u32x4_t, xf[buf][j]);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          v[k] &= (8 * h + 2 * k < left ? 0xffffu : 0u) | (8 * h + 2 * k + 1 < left ? 0xffff0000u : 0u);
        xf[buf][j] = __builtin_bit_cast(bf16x8_t, v);
      }
    }
    left -= 16;
    if (tile == 0)
      db += ((f[buf][0] + f[buf][1]) + (f[buf][2] + f[buf][3])) + ((f[buf][4] + f[buf][5]) + (f[buf][6] + f[buf][7]));
    bf16x8_t zf[3];
    split8(f[buf], zf);
#pragma unroll
    for (int n = 0; n < 3; ++n)
#pragma unroll
      for (int j = 0; j < NJ; ++j)
        acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xf[buf][j], zf[n], acc[j], 0, 0, 0);
  };
  pipeline_xk<St::NS, LOADS, kRgTok / 16>(q1 - q0, smem, St::BYTES / 2, issue, read, mma, [] {});

  if (tile == 0 && wn == 0) {
    const float s = db + __shfl_xor(db, 32, kWave);
    if (h == 0 && e_lane < E) a.db[(size_t)sp * E + e_lane] = s;
  }
  // rows of the tile are experts; columns past H (64 of the last tile's: H % 64 ==
  // 0) are not stored. At most 64 columns of a wave at a time go through LDS.
  constexpr int NE = NJ < 2 ? NJ : 2, EC = NE * 32;
  static_assert(W * 32 * EC * 4 <= St::BYTES * St::NS, "the epilogue's LDS");
#pragma unroll
  for (int j0 = 0; j0 < NJ; j0 += NE) {
    f32x16_t part[1][1][NE];
#pragma unroll
    for (int j = 0; j < NE; ++j) part[0][0][j] = acc[j0 + j];
    const int c = c0 + wn * WCOLS + j0 * 32;
    split_epilogue<1, NE, 1, 32, EC>(part, smem, 0, c < H ? E : 0, c, H, wm, 0, wave, lane,
                                     a.dw + (size_t)sp * E * H, 0, false);
  }
}

// Sums the S partial sums in order: 4 of 256 x 7168 (37 MB) 9.5 us, from the last-level
// cache.
__global__ __launch_bounds__(256) void router_dw_reduce_kernel(const float* __restrict__ part,
                                                               const float* __restrict__ pdb, int E, int H, int S,
                                                               float* __restrict__ dw, float* __restrict__ db) {
  const size_t n4 = (size_t)E * H / 4;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n4; i += (size_t)gridDim.x * 256)
    reinterpret_cast<float4*>(dw)[i] = sum_splits(part + i * 4, (size_t)E * H, S);
  for (int e = (int)(blockIdx.x * 256 + threadIdx.x); e < E; e += (int)gridDim.x * 256) {
    float s = 0.0f;
    for (int q = 0; q < S; ++q) s += pdb[(size_t)q * E + e];
    db[e] = s;
  }
}

// ---------------------------------------------------------------------------
// dx: a wave keeps the dz rows of its 32 tokens, in two terms, in registers (EP / 16
// fragments of either) and multiplies them with the columns of W that its block
// walks, 128 at a time; W comes to LDS in pieces of 64 experts x 128 columns by
// direct loads, NS pieces in a ring. Fragments of W are read one 16-expert step
// ahead of the MFMAs. Blocks that walk the same columns follow each other by the
// number of column ranges, so that (for 2, 4 or 8 of them) an XCD's L2 holds one or
// a few ranges of W. 16384 tokens, H = 7168, E = 256: 111-131 us (60 GFLOP, twice that
// on the MFMAs, and 235 MB written): 210 thousand cycles, MFMAs busy in 49 % of them,
// then the stores; 106 us at 2.2 GHz, in a row at what power leaves.
// ---------------------------------------------------------------------------
constexpr int kDxRows = 128;

template <int EP, bool VEC>
__global__ __launch_bounds__(256, 2) void router_dx_kernel(RouterGradArgs a, int tiles, int col_split) {
  constexpr int KC = EP / 64;                // pieces of a column tile
  constexpr int NS = 4;                      // pieces in the ring
  constexpr int STAGE = 64 * kRgCols;        // bf16
  constexpr int OUTB = 32 * 128;             // bytes of a wave's output rows, 64 columns at a time
  __shared__ __align__(16) bf16_t smem[NS * STAGE + 4 * OUTB / 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r32 = lane & 31, h = lane >> 5;
  const int E = a.E, H = a.H;
  const int part = (int)(blockIdx.x % (unsigned)col_split);
  const int row0 = uniform_int((int)(blockIdx.x / (unsigned)col_split) * kDxRows + wave * 32);
  const int tl0 = uniform_int(part * tiles / col_split);
  const int tl1 = uniform_int((part + 1) * tiles / col_split);
  bf16x8_t zf[EP / 16][2];
  {
    const float* p = a.dz + (size_t)min(row0 + r32, a.T - 1) * E;
#pragma unroll
    for (int s = 0; s < EP / 16; ++s) {
      const int e = 16 * s + 8 * h;
      float f[8];
      if (VEC) {
        const float4 u = e < E ? *reinterpret_cast<const float4*>(p + e) : make_float4(0, 0, 0, 0);
        const float4 v = e + 4 < E ? *reinterpret_cast<const float4*>(p + e + 4) : make_float4(0, 0, 0, 0);
        f[0] = u.x, f[1] = u.y, f[2] = u.z, f[3] = u.w, f[4] = v.x, f[5] = v.y, f[6] = v.z, f[7] = v.w;
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = e + k < E ? p[e + k] : 0.0f;
      }
      split8_nearest(f, zf[s]);
    }
  }
  // piece kc of column tile tl; 16 KB, 4 instructions a wave; rows past E read the last
  const int n = (tl1 - tl0) * KC;
  auto issue = [&](int q) {
    const int qq = q < n ? q : n - 1;
    const int tl = tl0 + qq / KC, kc = qq % KC;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = (i * 4 + wave) * 4 + lane / 16, e = min(kc * 64 + row, E - 1);
      const int c = min(tl * kRgCols + tr_swizzle(row, lane % 16) * 8, H - 8);
      dma16(a.w + (size_t)e * H + c, smem + (q % NS) * STAGE + (i * 4 + wave) * 512);
    }
  };
  wait_vmcnt<0>();
#pragma unroll
  for (int q = 0; q < NS - 1; ++q) issue(q);
  char* out = reinterpret_cast<char*>(smem + NS * STAGE) + wave * OUTB;
  // Stores of the tile before that were issued between the loads that a wait
  // counts: loads and stores leave the counter in the order of their issue.
  bool stored = false;
  for (int tl = tl0; tl < tl1; ++tl) {
    f32x16_t acc[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = f32x16_t{};
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      const int q = (tl - tl0) * KC + kc;
      wait_lgkmcnt0();  // this wave's reads of the piece before returned
      // piece q landed; younger are two pieces and, for the first three of a tile,
      // the eight stores of the tile before
      if (kc < 3 && stored)
        wait_vmcnt<4 * (NS - 2) + 8>();
      else
        wait_vmcnt<4 * (NS - 2)>();
      lds_barrier();
      issue(q + NS - 1);
      const char* base = reinterpret_cast<const char*>(smem + (q % NS) * STAGE);
      bf16x8_t wf[2][4];
#pragma unroll
      for (int j = 0; j < 4; ++j) wf[0][j] = tr_frag(base, lane, 0, j * 32);
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        if (s + 1 < 4)
#pragma unroll
          for (int j = 0; j < 4; ++j) wf[(s + 1) & 1][j] = tr_frag(base, lane, 16 * (s + 1), j * 32);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wf[s & 1][j], zf[kc * 4 + s][t], acc[j], 0, 0, 0);
      }
    }
    // lane (r, h) holds columns 8 g + 4 h + (0..3) of each 32 of its token: to whole
    // rows of 64 columns through the wave's LDS
    const bool whole = a.T - row0 >= 32 && (tl + 1) * kRgCols <= H;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      auto at = [](int r, int piece) { return r * 128 + ((piece ^ (r & 7)) * 16); };
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const f32x16_t& c = acc[half * 2 + j];
          *reinterpret_cast<uint2*>(out + at(r32, j * 4 + g) + h * 8) =
              make_uint2(pack_bf16x2(c[4 * g], c[4 * g + 1]), pack_bf16x2(c[4 * g + 2], c[4 * g + 3]));
        }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      const int col = tl * kRgCols + half * 64;
      u32x4_t v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const u32x4_t*>(out + at(i * 8 + lane / 8, lane % 8));
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      bf16_t* p = a.dx + (size_t)(row0 + lane / 8) * H + col + lane % 8 * 8;
      if (whole) {
#pragma unroll
        for (int i = 0; i < 4; ++i) *reinterpret_cast<u32x4_t*>(p + (size_t)i * 8 * H) = v[i];
      } else if (col < H) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (row0 + i * 8 + lane / 8 < a.T) *reinterpret_cast<u32x4_t*>(p + (size_t)i * 8 * H) = v[i];
      }
    }
    stored = whole;
  }
  wait_vmcnt<0>();
}

// ---------------------------------------------------------------------------
// fp32 (small layers): plain sums. 64 tokens, H = 128, E = 8: dW 4.2 us, dx 3.1 us,
// a launch and a chain of load latencies each.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(256) void router_dx_f32_kernel(const float* __restrict__ dz, const float* __restrict__ w,
                                                            int T, int E, int H, float* __restrict__ dx) {
  const size_t n = (size_t)T * H;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) {
    const size_t t = i / H;
    const int c = (int)(i - t * H);
    float s = 0.0f;
    for (int e = 0; e < E; ++e) s = fmaf(dz[t * E + e], w[(size_t)e * H + c], s);
    dx[i] = s;
  }
}

// Blocks of 64 columns x 8 experts x one range of tokens: a thread sums its column
// over every fourth token of the range (dz is the same in all lanes), and the four
// sums of a column are joined in LDS.
__global__ __launch_bounds__(256) void router_dw_f32_kernel(const float* __restrict__ dz, const float* __restrict__ x,
                                                            int T, int E, int H, int S, float* __restrict__ dw,
                                                            float* __restrict__ db) {
  __shared__ float s_sum[4][9][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tiles = (H + 63) / 64, eg = (E + 7) / 8;
  const int tile = (int)(blockIdx.x % (unsigned)tiles), r = (int)(blockIdx.x / (unsigned)tiles);
  const int e0 = r % eg * 8, sp = r / eg;
  const int c = tile * 64 + lane;
  const unsigned t0 = (unsigned)((long long)sp * T / S), t1 = (unsigned)((long long)(sp + 1) * T / S);
  float acc[8], sum[8];
#pragma unroll
  for (int q = 0; q < 8; ++q) acc[q] = sum[q] = 0.0f;
#pragma unroll 4
  for (unsigned t = t0 + wave; t < t1; t += 4) {  // unsigned: the last step passes T <= 2^31 - 1
    const float xv = c < H ? x[(size_t)t * H + c] : 0.0f;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const float d = dz[(size_t)t * E + min(e0 + q, E - 1)];
      acc[q] = fmaf(d, xv, acc[q]);
      sum[q] += d;
    }
  }
#pragma unroll
  for (int q = 0; q < 8; ++q) s_sum[wave][q][lane] = acc[q];
  if (lane == 0)
#pragma unroll
    for (int q = 0; q < 8; ++q) s_sum[wave][8][q] = sum[q];
  __syncthreads();
  auto join = [&](int q, int l) { return (s_sum[0][q][l] + s_sum[1][q][l]) + (s_sum[2][q][l] + s_sum[3][q][l]); };
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int q = wave * 2 + i, e = e0 + q;
    if (e < E && c < H) dw[((size_t)sp * E + e) * H + c] = join(q, lane);
  }
  if (tile == 0 && threadIdx.x < 8 && e0 + (int)threadIdx.x < E) db[(size_t)sp * E + e0 + threadIdx.x] = join(8, threadIdx.x);
}

// Blocks of router_dw_f32_kernel.
static unsigned dw_f32_grid(int E, int H, int S) { return (unsigned)((H + 63) / 64 * ((E + 7) / 8) * S); }

// Token ranges of dW: enough blocks for every CU, at least 64 tokens each.
static int router_ranges(int T, int E, int H, bool bf16) {
  const int cus = device_cu_count();
  const long long blocks = bf16 ? (H + kRgCols - 1) / kRgCols : dw_f32_grid(E, H, 1);
  const long long s = std::min(std::max(1LL, cus / blocks), std::max(1LL, T / 64LL));
  return (int)std::min(s, 64LL);
}

size_t router_grad_ws_bytes(int T, int E, int H, bool bf16) {
  const int S = router_ranges(T, E, H, bf16);
  return S > 1 ? round256((size_t)S * E * H * 4) + round256((size_t)S * E * 4) : 256;
}

hipError_t launch_router_grad(const float* dz, const void* x, const void* w, int T, int E, int H, bool bf16, void* dx,
                              float* dw, float* db, void* ws, hipStream_t s) {
  const int S = router_ranges(T, E, H, bf16);
  float* pw = S > 1 ? static_cast<float*>(ws) : dw;
  float* pb = S > 1 ? reinterpret_cast<float*>(static_cast<char*>(ws) + round256((size_t)S * E * H * 4)) : db;
  hipError_t e = hipSuccess;
  if (T == 0) {  // no tokens: dW and db are zero
    router_dw_f32_kernel<<<dw_f32_grid(E, H, 1), 256, 0, s>>>(dz, nullptr, 0, E, H, 1, dw, db);
    return hipGetLastError();
  }
  if (bf16) {
    RouterGradArgs a{dz, static_cast<const bf16_t*>(x), static_cast<const bf16_t*>(w), static_cast<bf16_t*>(dx),
                     pw, pb, T, E, H, S};
    const int tiles = (H + kRgCols - 1) / kRgCols;
    auto run = [&](auto ep, auto vec) {
      constexpr int EP = decltype(ep)::value;
      constexpr bool VEC = decltype(vec)::value;
      router_dw_kernel<EP, VEC><<<(unsigned)(tiles * S), 512, 0, s>>>(a);
      e = hipGetLastError();
      if (e != hipSuccess || dx == nullptr) return;
      const int rows = (T - 1) / kDxRows + 1;
      const int split = std::min(tiles, std::max(1, (2 * device_cu_count() + rows - 1) / rows));
      router_dx_kernel<EP, VEC><<<(unsigned)(rows * split), 256, 0, s>>>(a, tiles, split);
      e = hipGetLastError();
    };
    auto by_vec = [&](auto ep) {
      if (E % 4 == 0)
        run(ep, std::true_type());
      else
        run(ep, std::false_type());
    };
    if (E <= 64)
      by_vec(std::integral_constant<int, 64>());
    else if (E <= 128)
      by_vec(std::integral_constant<int, 128>());
    else
      by_vec(std::integral_constant<int, 256>());
  } else {
    auto grid = [](size_t n) { return (unsigned)std::min<size_t>((n + 255) / 256, 1u << 16); };
    router_dw_f32_kernel<<<dw_f32_grid(E, H, S), 256, 0, s>>>(dz, static_cast<const float*>(x), T, E, H, S, pw, pb);
    e = hipGetLastError();
    if (e == hipSuccess && dx != nullptr) {
      router_dx_f32_kernel<<<grid((size_t)T * H), 256, 0, s>>>(dz, static_cast<const float*>(w), T, E, H,
                                                               static_cast<float*>(dx));
      e = hipGetLastError();
    }
  }
  if (e != hipSuccess || S == 1) return e;
  router_dw_reduce_kernel<<<(unsigned)(4 * device_cu_count()), 256, 0, s>>>(pw, pb, E, H, S, dw, db);
  return hipGetLastError();
}

}  // namespace moe
