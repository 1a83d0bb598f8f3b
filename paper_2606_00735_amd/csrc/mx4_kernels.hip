// MXFP4 (OCP MX block scaling with E2M1 elements, mx.hpp): quantisation of
// activations and expert weights, the values of codes, and the expert FFN on
// 4-bit operands.
#include <algorithm>

#include "common.hpp"
#include "grouped_gemm.hpp"
#include "launch.hpp"
#include "mx.hpp"

namespace moe {

// ---------------------------------------------------------------------------
// Quantisation: x [batch][rows][K] (bf16 or fp32) -> codes (rows ldc bytes
// apart) and scale dwords [batch][chunks][rows][2].
//
// Bound by the copy: a row's chunk of 256 elements is 512 bytes of bf16 (1 KB
// of fp32) in, one 128-byte line of codes and 8 bytes of scales out. A block
// takes kQRows rows x kQChunks chunks, so that the scales of a chunk leave as
// whole lines (16 rows x 8 bytes) and every thread has kQChunks * 2 loads in
// flight. 32 lanes work on a row's chunk, 8 elements each: the 4 lanes of a
// block find its largest magnitude with two shuffles. 16384 x 7168 bf16 (297 MB):
// 62-67 us, 4.4-4.8 TB/s (a 2 GiB copy: 4.76); 333 x 4224 fp32 3.8 us, a launch and
// two latencies.
// row_count (device, optional, batch 1 only): only rows [0, min(rows,
// *row_count)) are quantised; the others are left as they are.
// ---------------------------------------------------------------------------
constexpr int kQRows = 16, kQChunks = 2;

// A block's share: kQRows rows from row0 on of matrix b, kQChunks chunks from
// chunk0 on. Fewer than 2^32 - 2^20 of them, so that a block's step past the last does
// not wrap: K <= 512 is one group of chunks, rows <= 16 one of rows, and batch * rows * K
// <= 2^40 with batch < 2^31 leaves at most 4.05e9 (17 rows of K = 32).
struct QTile {
  size_t b;
  int row0, chunk0;
};
__host__ __device__ __forceinline__ uint32_t q_cgroups(int K) {
  return (uint32_t)((K + kMx4Chunk * kQChunks - 1) / (kMx4Chunk * kQChunks));
}
__host__ __device__ __forceinline__ uint32_t q_rgroups(int rows) {
  return ((uint32_t)rows + kQRows - 1) / kQRows;
}
__device__ __forceinline__ QTile q_tile(uint32_t u, int rows, int K) {
  const uint32_t ncg = q_cgroups(K), nrg = q_rgroups(rows);
  const uint32_t r = u / ncg, b = r / nrg;
  return {b, (int)((r - b * nrg) * kQRows), (int)((u - r * ncg) * kQChunks)};
}
constexpr uint32_t kQMaxGrid = 1u << 20;  // blocks of a launch; each loops over the rest

template <bool F32IN>
__global__ __launch_bounds__(256) void mx4_quantize_kernel(const void* __restrict__ x, uint32_t tiles, int rows,
                                                           int K, int ldc, const int32_t* __restrict__ row_count,
                                                           uint8_t* __restrict__ codes,
                                                           uint32_t* __restrict__ scales) {
  const int live = row_count != nullptr ? min(max(*row_count, 0), rows) : rows;
  const int chunks = (K + kMx4Chunk - 1) / kMx4Chunk;
  const int lane32 = threadIdx.x & 31, group = threadIdx.x >> 5;  // 8 groups of 32 lanes
  constexpr int NT = kQRows * kQChunks / 8;                       // (row, chunk) pairs of a group
  for (uint32_t u0 = blockIdx.x; u0 < tiles; u0 += gridDim.x) {
    const QTile tile = q_tile(u0, rows, K);
    const size_t b = tile.b;
    uint32_t v[NT][8];  // fp32 bits
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int p = i * 8 + group, row = tile.row0 + p / kQChunks;
      const int col = (tile.chunk0 + p % kQChunks) * kMx4Chunk + lane32 * 8;
      const bool in = row < live && col < K;
      const size_t off = in ? (b * rows + row) * (size_t)K + col : 0;
      if (F32IN) {
        const uint4* s = reinterpret_cast<const uint4*>(static_cast<const float*>(x) + off);
        uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
        if (in) lo = s[0], hi = s[1];
        v[i][0] = lo.x, v[i][1] = lo.y, v[i][2] = lo.z, v[i][3] = lo.w;
        v[i][4] = hi.x, v[i][5] = hi.y, v[i][6] = hi.z, v[i][7] = hi.w;
      } else {
        uint4 u = make_uint4(0, 0, 0, 0);
        if (in) u = *reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(x) + off);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) v[i][2 * q] = w[q] << 16, v[i][2 * q + 1] = w[q] & 0xFFFF0000u;
      }
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int p = i * 8 + group, row = tile.row0 + p / kQChunks, chunk = tile.chunk0 + p % kQChunks;
      uint32_t top = 0;
#pragma unroll
      for (int q = 0; q < 8; ++q) top = max(top, v[i][q] & 0x7fffffffu);
      top = max(top, (uint32_t)__shfl_xor((int)top, 1, kWave));
      top = max(top, (uint32_t)__shfl_xor((int)top, 2, kWave));
      const uint32_t code = mx4_scale_code(top);
      const float sc = mx4_scale(code);
      auto f = [&](int q) { return __uint_as_float(v[i][q]); };
      uint32_t out = e2m1x4(f(0), f(1), f(2), f(3), sc) | e2m1x4(f(4), f(5), f(6), f(7), sc) << 16;
      if (code == kMxNan) out = 0;
      // lane h of the first two gathers the codes of blocks h, 2 + h, 4 + h, 6 + h
      uint32_t word = 0;
      const int h = lane32 & 1;
#pragma unroll
      for (int s = 0; s < 4; ++s) word |= (uint32_t)__shfl((int)code, (2 * s + h) * 4, 32) << (8 * s);
      if (row < live && chunk < chunks) {
        *reinterpret_cast<uint32_t*>(codes + (b * rows + row) * (size_t)ldc + chunk * 128 + lane32 * 4) = out;
        if (lane32 < 2) scales[((b * chunks + chunk) * rows + row) * 2 + lane32] = word;
      }
    }
  }
}

hipError_t launch_mx4_quantize(const void* x, bool f32, int batch, int rows, int K, int ldc,
                               const int32_t* row_count, uint8_t* codes, uint32_t* scales, hipStream_t s) {
  const uint32_t tiles = (uint32_t)batch * q_rgroups(rows) * q_cgroups(K), grid = std::min(tiles, kQMaxGrid);
  if (f32)
    mx4_quantize_kernel<true><<<grid, 256, 0, s>>>(x, tiles, rows, K, ldc, row_count, codes, scales);
  else
    mx4_quantize_kernel<false><<<grid, 256, 0, s>>>(x, tiles, rows, K, ldc, row_count, codes, scales);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// The values that codes stand for, exact in bf16 (two significant bits under a
// power of two of at least 2^-128). The tiling of the quantiser: a group of 32
// lanes reads a row's chunk, 4 bytes a lane, and writes its 512 bytes. Bound by the
// stores: 16384 x 7168 (297 MB) 66-70 us, 4.2-4.5 TB/s.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(256) void mx4_dequantize_kernel(const uint8_t* __restrict__ codes,
                                                             const uint8_t* __restrict__ scales, uint32_t tiles,
                                                             int rows, int K, int ldc, bf16_t* __restrict__ x) {
  const int chunks = (K + kMx4Chunk - 1) / kMx4Chunk;
  const int lane32 = threadIdx.x & 31, group = threadIdx.x >> 5;
  constexpr int NT = kQRows * kQChunks / 8;
  for (uint32_t u0 = blockIdx.x; u0 < tiles; u0 += gridDim.x) {
    const QTile tile = q_tile(u0, rows, K);
    const size_t b = tile.b;
    uint32_t w[NT], c[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int p = i * 8 + group, row = tile.row0 + p / kQChunks, chunk = tile.chunk0 + p % kQChunks;
      const bool in = row < rows && chunk * kMx4Chunk + lane32 * 8 < K;
      w[i] = c[i] = 0;
      if (in) {
        w[i] = *reinterpret_cast<const uint32_t*>(codes + (b * rows + row) * (size_t)ldc + chunk * 128 + lane32 * 4);
        c[i] = scales[((b * chunks + chunk) * rows + row) * 8 + mx4_scale_byte(lane32 >> 2)];
      }
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int p = i * 8 + group, row = tile.row0 + p / kQChunks, chunk = tile.chunk0 + p % kQChunks;
      const int col = chunk * kMx4Chunk + lane32 * 8;
      if (row >= rows || col >= K) continue;
      uint32_t o[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t r = 0;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t n = (w[i] >> (8 * q + 4 * e)) & 15u;
          // bf16 bits of the E2M1 value: 0, 0.5, or exponent and mantissa bit
          // moved to place (exponent bias 1 -> 127, mantissa to the top bit)
          const uint32_t m = n & 7u;
          float f = m < 2u ? (m ? 0.5f : 0.0f) : __uint_as_float(((m >> 1) + 126u) << 23 | (m & 1u) << 22);
          f = ldexpf(f, (int)c[i] - 127);
          if (c[i] == kMxNan) f = __uint_as_float(0x7fc00000u);
          r |= (__float_as_uint(f) >> 16 | (n & 8u) << 12) << (16 * e);
        }
        o[q] = r;
      }
      *reinterpret_cast<uint4*>(x + (b * rows + row) * (size_t)K + col) = make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
}

hipError_t launch_mx4_dequantize(const uint8_t* codes, const uint32_t* scales, int batch, int rows, int K, int ldc,
                                 void* x, hipStream_t s) {
  const uint32_t tiles = (uint32_t)batch * q_rgroups(rows) * q_cgroups(K);
  mx4_dequantize_kernel<<<std::min(tiles, kQMaxGrid), 256, 0, s>>>(
      codes, reinterpret_cast<const uint8_t*>(scales), tiles, rows, K, ldc,
                                             static_cast<bf16_t*>(x));
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Expert FFN: gate/up (MXFP4 in, MXFP4 h out), then down (bf16 out), by the tile
// schedules of the bf16 FFN (grouped_gemm.hpp).
//
// Measured, gate/up + down: decode (8 experts of 8 rows, H = 4096, I = 14336, 749 MB
// of weights) 92 + 47 us, 5.4 TB/s, the memory's streaming rate (95 L1 misses in flight
// a CU); 128 experts of about 60 rows (H = 2048, I = 768) 62 + 41 us, 3.1 TB/s: the
// pipelines' fills and the epilogues of K loops of 8 and of 3 chunks (56 and 40 misses
// in flight); prefill (8192 rows, H = 4096, I = 14336) 620-665 + 280-303 us and their
// reductions' 20 us, 3.0 PFLOP/s: MFMAs busy 39 % of the cycles of gate/up and 40 % of
// down, the rest the LDS and issue of the K loop and what stands around it, as follows;
// the cycles are the same at a clock of 2.2 GHz (547 + 267 us, launches with pauses
// between them) and at the lower one that power leaves to launches in a row.
// ---------------------------------------------------------------------------
// 8 waves for every tile: the 256-row tile in quadrant phases on 4 waves that bf16
// and MXFP8 take for large experts was no faster at 4 bits (FFN us, 4 / 8 waves, 8
// experts of 1024 rows, H = 4096, I = 14336: 891 / 893; 32 of 512 rows, H = 7168, I =
// 2048: 597 / 587; 128 of 512 rows, H = 2048, I = 768: 353 / 353). A tile's K loop is
// a quarter as long, and what stands around it counts for more: per 256 x 256 tile a
// product of 8192 x 8192 over K took 14.5 us + K / 16384 x 102 us (5.4 PFLOP/s in
// the loop), the dual one 10.6 + K / 16384 x 112 us: the outputs' stores (128 KB a CU
// at once, 7 us at the memory's rate) and SiLU and quantisation (1250 vector and 256
// transcendental instructions a wave, 5 us). Loading the next tile's first chunks
// before the epilogue gained nothing (888 / 890): the K loop's waits then count the
// stores, which leave the counter in order.
template <bool DUAL>
__global__ __launch_bounds__(8 * kWave) void grouped_gemm_mx4_kernel(GemmArgs a) {
  grouped_gemm_body<8, DUAL, kMx4>(a);
}

// The MXFP4 gate/up reduction: sums the S partials of gate and up for 4
// consecutive columns of a row per thread in split order, applies SiLU(gate) * up
// and quantises each 32-column block (the 8 lanes of an aligned lane group; N % 32
// == 0 keeps a group inside one block and wholly in range or out). Does nothing
// when the GEMM before it split nothing.
__global__ __launch_bounds__(256) void split_reduce_mx4_kernel(GemmArgs a) {
  const int32_t* plan = a.plan;
  const int S = plan[0], N = a.N;
  if (S <= 1) {  // tail tiles of an unsplit launch
    const int St = plan[2];
    if (St <= 1) return;
    const size_t items = (size_t)plan[3] * 256 * (plan[4] / 4);
    for (size_t it = (size_t)blockIdx.x * 256 + threadIdx.x; it < items; it += (size_t)gridDim.x * 256) {
      TailItem t;
      if (!tail_item(a.part, plan, 2, it, t)) continue;
      const float4 g = sum_splits(t.p, t.tsz, St), u = sum_splits(t.p + St * t.tsz, t.tsz, St);
      mx4_quant_store4(a, silu_mul_fast(g.x, u.x), silu_mul_fast(g.y, u.y), silu_mul_fast(g.z, u.z),
                       silu_mul_fast(g.w, u.w), t.row, t.col);
    }
    return;
  }
  const int R = plan[1], n4 = N / 4;
  const size_t items = (size_t)R * n4, sstride = (size_t)R * N, bstride = (size_t)S * R * N;
  for (size_t it = (size_t)blockIdx.x * 256 + threadIdx.x; it < items; it += (size_t)gridDim.x * 256) {
    const int j = (int)(it / n4), c = (int)(it % n4) * 4;
    const float* p = a.part + (size_t)j * N + c;
    const float4 g = sum_splits(p, sstride, S), u = sum_splits(p + bstride, sstride, S);
    mx4_quant_store4(a, silu_mul_fast(g.x, u.x), silu_mul_fast(g.y, u.y), silu_mul_fast(g.z, u.z),
                     silu_mul_fast(g.w, u.w), plan[kPlanHead + j], c);
  }
}

// ---------------------------------------------------------------------------
// The FFN of few rows (a token's experts): latency. No LDS ring, no partial sums
// across blocks: a block takes 16 rows of an expert by 64 weight rows (32 columns of
// gate and up, or 64 of down), its 8 waves 32 weight rows x a quarter of K each,
// straight from memory to the operand registers of the 16 x 16 x 128 MFMA, kFewBatch
// chunks of a row a step; the quarters' sums meet in LDS, in order. Every wave finds
// the block's expert itself, from the offsets.
//
// Bound by the latency of offsets, rows and weights, one after the other, 5 us a
// launch (7 with cold operands); by the load path of the CUs that have a block when
// there are few; by memory from some 100 MB on, where the decode schedule's ring keeps
// more in flight. FFN us (bytes of the gate/up codes), the decode schedule / this: H =
// 2048, I = 768, 8 experts of 1 row (13 MB) 22.4 / 10.9, 32 of 2 (50 MB) 28.1 / 23.5, 64
// of 1 (101 MB) 45.4 / 41.8, 128 of 8 (201 MB) 81 / 84, 16 of 64 29.5 / 45.2; H = 7168,
// I = 2048, 1 of 1 (15 MB) 21.0 / 17.1, 1 of 64 31.4 / 24.1, 1 of 128 43.4 / 40.1, 8 of 1
// (117 MB) 52.6 / 45.7, 8 of 14 57.8 / 64.5, 32 of 4 (470 MB) 153 / 166; H = 4096, I =
// 14336, 1 of 1 (59 MB) 32.2 / 33.0, 2 of 60 62.9 / 171, 8 of 8 (470 MB) 146 / 175.
// The rule takes each product by itself, so that the halves of a call may differ (us, the
// decode schedule for both / as chosen / this for both, in a graph): H = 2048, I = 768,
// 96 rows on 70 of 128 experts 58 / 53 / 48, 128 rows on 86 67 / 59 / 55; H = 7168, I = 2048,
// 32 experts, two of them with a row of 16 that they might have 29 / 23 / 21, and where
// 32 and 128 rows might be there but 5 and 18 are, 41 / 41 / 36 and 84 / 85 / 88; H = 5120, I
// = 8192, 16 experts, one row of 4 32 / 30 / 27, 15 of 64 128 / 129 / 147. It counts the
// rows that may be there, not those that are, and so gives some away on a shard.
// A step of two chunks instead of four: 17.3 for 16.9, 46.1 for 45.7. At most 80
// registers, so that a CU holds three blocks: 64 experts of 1 row 41.8 for 44.0 with
// two; with 64 registers (four blocks, some spilt) 56, with all of a step's loads issued
// before its first product (160 registers, one block) 79.
// ---------------------------------------------------------------------------
constexpr int kFewTile = 16;   // rows of a tile
constexpr int kFewSplit = 4;   // parts of K
constexpr int kFewBatch = 4;   // chunks of a wave's step

// Sum of x over this lane and the lanes below.
__device__ __forceinline__ int lane_prefix(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // lane 15 to the next row of 16
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // lane 31 to the upper 32
  return x;
}

template <bool DUAL>
__global__ __launch_bounds__(8 * kWave, 6) void mx4_few_rows_kernel(GemmArgs a) {
  constexpr int COLS = DUAL ? 32 : 64, Q = kMaxExperts / kWave;
  __shared__ f32x4_t s_sum[8][2][kWave];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int cg = wave & 1, ks = wave >> 1;  // columns, part of K
  const int r16 = lane & 15, g = lane >> 4;
  const int E = a.E_local, N = a.N, K = a.K, nK = K / kMxChunk;

  // row tiles of the experts up to lane's (q * 64 + lane), clamped as in grouped_gemm_body
  int row0[Q], rows[Q], upto[Q];
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    const int e = q * kWave + lane;
    const int o0 = a.offsets[min(e, E)], o1 = a.offsets[min(e + 1, E)];
    row0[q] = min(max(o0, 0), a.M_cap);
    rows[q] = e < E ? min(max(o1, row0[q]), a.M_cap) - row0[q] : 0;
  }
  int total = 0;
#pragma unroll
  for (int q = 0; q < Q; ++q) {
    upto[q] = total + lane_prefix((rows[q] + kFewTile - 1) / kFewTile);
    total = __builtin_amdgcn_readlane(upto[q], kWave - 1);
  }
  const unsigned ct = (unsigned)N / COLS;
  const bool gather = a.a_src != nullptr;
  const size_t sa_rows = gather ? (size_t)a.a_T : (size_t)a.M_cap;
  for (unsigned item = blockIdx.x; item < (unsigned)total * ct; item += gridDim.x) {
    const int j = uniform_int((int)(item / ct)), n0 = (int)(item - (unsigned)j * ct) * COLS;
    int e = 0;
#pragma unroll
    for (int q = 0; q < Q; ++q) e += (int)__popcll(__ballot(upto[q] <= j));
    e = uniform_int(e);
    int m0 = 0, n_rows = 0, before = 0;
#pragma unroll
    for (int q = 0; q < Q; ++q)
      if (e / kWave == q) {
        m0 = __builtin_amdgcn_readlane(row0[q], e % kWave);
        n_rows = __builtin_amdgcn_readlane(rows[q], e % kWave);
        before = __builtin_amdgcn_readlane(upto[q], e % kWave) - (n_rows + kFewTile - 1) / kFewTile;
      }
    const int skip = (j - before) * kFewTile;
    m0 += skip, n_rows = min(n_rows - skip, kFewTile);

    // Piece 4 t + g of a row's chunk for k-step t; its scale is byte 2 t + g / 2 of
    // dword g % 2.
    const int m = m0 + min(r16, n_rows - 1);
    const int row = gather ? min(max(a.a_src[m] / a.a_div, 0), a.a_T - 1) : m;
    const uint32_t offB = (uint32_t)(r16 * a.ldb + g * 16), offSB = (uint32_t)(r16 * 2 + (g & 1));
    const char *B[2], *A = reinterpret_cast<const char*>(a.A) + (size_t)row * K + g * 16;
    const uint32_t *SB[2], *SA = a.As + (size_t)row * 2 + (g & 1);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const size_t n = n0 + (DUAL ? cg * 16 : cg * 32 + b * 16);
      B[b] = reinterpret_cast<const char*>(DUAL && b ? a.B1 : a.B0) + ((size_t)e * N + n) * a.ldb;
      SB[b] = (DUAL && b ? a.Bs1 : a.Bs0) + ((size_t)e * nK * N + n) * 2;
    }
    f32x4_t acc[2] = {f32x4_t{}, f32x4_t{}};
    const int c_end = (ks + 1) * nK / kFewSplit;
#pragma unroll 1
    for (int c = ks * nK / kFewSplit; c < c_end; c += kFewBatch) {
      uint4 w[kFewBatch][2][2], x[kFewBatch][2];
      uint32_t sw[kFewBatch][2], sx[kFewBatch];
#pragma unroll
      for (int u = 0; u < kFewBatch; ++u) {
        const size_t cc = (size_t)min(c + u, c_end - 1);  // past the part: a repeated, unused load
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
          for (int t = 0; t < 2; ++t) w[u][b][t] = *reinterpret_cast<const uint4*>(B[b] + cc * 128 + t * 64 + offB);
          sw[u][b] = SB[b][cc * N * 2 + offSB];
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) x[u][t] = *reinterpret_cast<const uint4*>(A + cc * 128 + t * 64);
        sx[u] = SA[cc * sa_rows * 2];
      }
#pragma unroll
      for (int u = 0; u < kFewBatch; ++u) {
        if (c + u >= c_end) break;
        const uint32_t sa = sx[u] >> (8 * (g >> 1));
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const uint32_t sb = sw[u][b] >> (8 * (g >> 1));
          acc[b] = mfma_mx4_16<0>(w[u][b][0], x[u][0], acc[b], sb, sa);
          acc[b] = mfma_mx4_16<2>(w[u][b][1], x[u][1], acc[b], sb, sa);
        }
      }
    }
    // lane (r, g) holds columns 4 g + (0..3) of row r
    s_sum[wave][0][lane] = acc[0];
    s_sum[wave][1][lane] = acc[1];
    __syncthreads();
    auto sum = [&](int half, int b, int at) {
      f32x4_t s = s_sum[half][b][at];
#pragma unroll
      for (int p = 1; p < kFewSplit; ++p) s += s_sum[p * 2 + half][b][at];
      return s;
    };
    if constexpr (DUAL) {
      const int r = tid >> 3, c4 = tid & 7, at = (c4 & 3) * 16 + r;
      if (r < n_rows) {
        const f32x4_t gt = sum(c4 >> 2, 0, at), up = sum(c4 >> 2, 1, at);
        mx4_quant_store4(a, silu_mul_fast(gt[0], up[0]), silu_mul_fast(gt[1], up[1]), silu_mul_fast(gt[2], up[2]),
                         silu_mul_fast(gt[3], up[3]), m0 + r, n0 + c4 * 4);
      }
    } else {
      const int r = tid >> 4, c4 = tid & 15;
      if (r < n_rows) {
        const f32x4_t v = sum(c4 >> 3, (c4 >> 2) & 1, (c4 & 3) * 16 + r);
        *reinterpret_cast<uint2*>(a.C + (size_t)(m0 + r) * N + n0 + c4 * 4) =
            make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
      }
    }
    __syncthreads();  // before the next item's sums
  }
}

// Row tiles that `rows` rows of E_local experts can make, at most.
static int few_tiles(int rows, int E_local) {
  const int n = std::min(rows, E_local);
  return n + (rows - n) / kFewTile;
}
// Whether a launch takes it: at most kFewRows rows and, however they fall on the
// experts, kFewBytes of weight codes, an expert's as often as it has row tiles.
constexpr int kFewRows = 128;
constexpr long long kFewBytes = 128LL << 20;
static bool few_rows(int rows, int E_local, int N, int K, int matrices) {
  return rows <= kFewRows && (long long)few_tiles(rows, E_local) * N * mx4_row_bytes(K) * matrices <= kFewBytes;
}
static unsigned few_grid(int rows, int E_local, int N, int cols) {
  return (unsigned)std::min<long long>((long long)few_tiles(rows, E_local) * (N / cols), 8LL * device_cu_count());
}

// Workspace: counters (kCntBytes, zero before first use, as for bf16) | h codes
// [M_cap][row bytes of I] | h scale dwords [chunks of I][M_cap][2] | split-K plan
// | fp32 partials (split-K, or the decode schedule's slots).
struct FfnMx4Ws {
  size_t hq, hs, plan, part;  // byte offsets
  long long part_cap;
  int plan_rows;
  size_t bytes;
};

static FfnMx4Ws ffn_mx4_ws_layout(int M_cap, int E_local, int H, int I) {
  FfnMx4Ws w{};
  const size_t ib = (size_t)mx4_row_bytes(I);
  w.hq = kCntBytes;
  w.hs = w.hq + round256(M_cap * ib);
  w.plan = w.hs + round256(ib / 128 * M_cap * 8);
  const long long need = (long long)kMaxSplit * M_cap * std::max(2LL * I, (long long)H);
  w.part_cap = std::min(need, kPartCapFloats);
  w.plan_rows = std::max(M_cap, kSmallM * E_local);
  w.part = w.plan + round256((size_t)(kPlanHead + (size_t)w.plan_rows) * 4);
  w.bytes = w.part + round256((size_t)std::max(w.part_cap, sk_slot_floats()) * 4);
  return w;
}

size_t ffn_mx4_ws_bytes(int M_cap, int E_local, int H, int I) {
  return ffn_mx4_ws_layout(M_cap, E_local, H, I).bytes;
}

static hipError_t gateup_mx4(const Mx4Rows& x, const Mx4Weights& wg, const Mx4Weights& wu, const int32_t* offsets,
                             int E_local, int H, int I, int M_cap, uint8_t* hq, uint32_t* hs, const MxSplit& sp,
                             hipStream_t s) {
  GemmArgs g{};
  g.A = reinterpret_cast<const bf16_t*>(x.codes);
  g.B0 = reinterpret_cast<const bf16_t*>(wg.codes);
  g.B1 = reinterpret_cast<const bf16_t*>(wu.codes);
  g.C = reinterpret_cast<bf16_t*>(hq);
  g.offsets = offsets;
  g.E_local = E_local;
  g.M_cap = M_cap;
  g.N = I;
  g.K = mx4_row_bytes(H);
  g.ldb = wg.ld;
  g.a_src = x.src;
  g.a_div = x.div;
  g.a_T = x.T;
  mx_split_args(g, sp);
  g.As = x.scales;
  g.Bs0 = wg.scales;
  g.Bs1 = wu.scales;
  g.Cs = hs;
  if (few_rows(M_cap, E_local, I, H, 2)) {
    mx4_few_rows_kernel<true><<<few_grid(M_cap, E_local, I, 32), 8 * kWave, 0, s>>>(g);
    return hipGetLastError();
  }
  const bool split = sp.plan != nullptr && g.K / kMxChunk >= 2 * kMinSplitChunks;
  grouped_gemm_mx4_kernel<true><<<mx_grid(M_cap, E_local, I, split || g.sk), 8 * kWave, 0, s>>>(g);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !split || sp.no_reduce) return e;
  split_reduce_mx4_kernel<<<mx_reduce_grid(0, 0), 256, 0, s>>>(g);
  return hipGetLastError();
}

static hipError_t gemm_mx4(const uint8_t* aq, const uint32_t* as, const Mx4Weights& w, const int32_t* offsets,
                           int E_local, int N, int K, int M_cap, void* c, const MxSplit& sp, hipStream_t s) {
  GemmArgs g{};
  g.A = reinterpret_cast<const bf16_t*>(aq);
  g.B0 = reinterpret_cast<const bf16_t*>(w.codes);
  g.C = static_cast<bf16_t*>(c);
  g.offsets = offsets;
  g.E_local = E_local;
  g.M_cap = M_cap;
  g.N = N;
  g.K = mx4_row_bytes(K);
  g.ldb = w.ld;
  mx_split_args(g, sp);
  g.As = as;
  g.Bs0 = w.scales;
  if (few_rows(M_cap, E_local, N, K, 1)) {
    mx4_few_rows_kernel<false><<<few_grid(M_cap, E_local, N, 64), 8 * kWave, 0, s>>>(g);
    return hipGetLastError();
  }
  const bool split = sp.plan != nullptr && g.K / kMxChunk >= 2 * kMinSplitChunks;
  grouped_gemm_mx4_kernel<false><<<mx_grid(M_cap, E_local, N, split || g.sk), 8 * kWave, 0, s>>>(g);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !split || sp.no_reduce) return e;
  split_reduce_kernel<false><<<mx_reduce_grid(0, 0), 256, 0, s>>>(sp.part, sp.plan, N, static_cast<bf16_t*>(c));
  return hipGetLastError();
}

hipError_t launch_gateup_mx4(const Mx4Rows& x, const Mx4Weights& wg, const Mx4Weights& wu, const int32_t* offsets,
                             int E_local, int H, int I, int M_cap, uint8_t* hq, uint32_t* hs, hipStream_t s) {
  if (E_local == 0 || M_cap == 0) return hipSuccess;
  return gateup_mx4(x, wg, wu, offsets, E_local, H, I, M_cap, hq, hs, MxSplit{}, s);
}

hipError_t launch_gemm_mx4(const uint8_t* aq, const uint32_t* as, const Mx4Weights& w, const int32_t* offsets,
                           int E_local, int N, int K, int M_cap, void* c, hipStream_t s) {
  if (E_local == 0 || M_cap == 0) return hipSuccess;
  return gemm_mx4(aq, as, w, offsets, E_local, N, K, M_cap, c, MxSplit{}, s);
}

hipError_t launch_ffn_mx4(const Mx4Rows& x, const Mx4Weights& wg, const Mx4Weights& wu, const Mx4Weights& wd,
                          const int32_t* offsets, int E_local, int H, int I, int M_cap, void* y_perm, void* ws,
                          hipStream_t s) {
  if (E_local == 0 || M_cap == 0) return hipSuccess;
  const FfnMx4Ws L = ffn_mx4_ws_layout(M_cap, E_local, H, I);
  char* w = static_cast<char*>(ws);
  uint8_t* hq = reinterpret_cast<uint8_t*>(w + L.hq);
  uint32_t* hs = reinterpret_cast<uint32_t*>(w + L.hs);
  int32_t* cnt = reinterpret_cast<int32_t*>(w);
  // as in launch_ffn: a token adds at most one row to an expert, so with the
  // row gather the bound on an expert's rows is min(T, M_cap)
  const bool no_reduce = (x.src != nullptr ? std::min(x.T, M_cap) : M_cap) <= kSkHostRows;
  const MxSplit sp1{reinterpret_cast<float*>(w + L.part), L.part_cap, reinterpret_cast<int32_t*>(w + L.plan),
                    L.plan_rows, cnt + kQueueGU, cnt + kDoneGU, cnt + kTcntGU, no_reduce, xcd_state(s)};
  hipError_t e = gateup_mx4(x, wg, wu, offsets, E_local, H, I, M_cap, hq, hs, sp1, s);
  if (e != hipSuccess) return e;
  const MxSplit sp2{sp1.part, sp1.part_cap, sp1.plan, sp1.plan_rows, cnt + kQueueDN, cnt + kDoneDN, cnt + kTcntDN,
                    no_reduce, sp1.xcd};
  return gemm_mx4(hq, hs, wd, offsets, E_local, H, I, M_cap, y_perm, sp2, s);
}

}  // namespace moe
