// Dense products with an epilogue, and their gradients (gfx950):
//   y  = act(x w^T + bias) * mul + residual
//   dz = dy * mul * act'(z), dx = dz w, dw = dz^T x, dbias = sum of dz's rows
//
// All three products are C[rows, cols] = sum over k of A(row, k) B(col, k), k the
// reduction: x and w have it along their rows; w in dx and both operands of dw have it
// as their row index ("transposed" below). A transposed operand is copied to LDS as it
// lies in memory and its fragments are read with the transposing read, so that no
// operand is ever laid out anew. Sums are fp32 in the MFMA; a result is rounded once.
#include <algorithm>
#include <climits>
#include <type_traits>

#include "common.hpp"
#include "grouped_gemm.hpp"
#include "launch.hpp"

namespace moe {

namespace {

typedef short s16x4_t __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------
// Activations, fp32.
// ---------------------------------------------------------------------------
__device__ __forceinline__ float sigmoid32(float z) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-z * 1.4426950408889634f));
}
// exp(-z^2 / 2)
__device__ __forceinline__ float bell(float z) { return __builtin_amdgcn_exp2f(z * z * -0.7213475204f); }
// The normal distribution's integral up to z. Its small side is exp(-z^2 / 2) R(|z|), R
// smooth: a polynomial of degree 8 in t = 1 / (1 + 0.3 |z|), fitted for the least largest
// relative error over [0, 14], 1.7e-7 with its constants in fp32, 4.8e-7 computed in fp32 (a call of erfcf cost an epilogue of
// 16384 x 2048 values 50 us).
__device__ __forceinline__ float normal_below(float z) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.3f, fabsf(z), 1.0f));
  float p = 0.03567765653133392f;
  p = fmaf(p, t, -0.15721559524536133f);
  p = fmaf(p, t, 0.20637577772140503f);
  p = fmaf(p, t, -0.05370469018816948f);
  p = fmaf(p, t, 0.1285729855298996f);
  p = fmaf(p, t, 0.09990999847650528f);
  p = fmaf(p, t, 0.12075452506542206f);
  p = fmaf(p, t, 0.11962926387786865f);
  const float q = p * t * bell(z);
  return z >= 0.0f ? 1.0f - q : q;
}

// F32: the data are fp32, whose silu is to be exact at any size of z (5 u of the value, a step being
// 2 u): by an exponential of -|z| itself, which neither overflows nor rounds its argument, and true
// quotients. Of bf16 data a value is rounded by up to 2^-8 of itself; sigmoid32's argument, rounded
// before the exponential, moves it by |z| 2^-24.
template <int ACT, bool F32 = false>
__device__ __forceinline__ float act_value(float z) {
  if (ACT == kActRelu) return z < 0.0f ? 0.0f : z;
  if (ACT == kActSilu && F32) {
    const float e = expf(-fabsf(z));
    return (z < 0.0f ? z * e : z) / (1.0f + e);
  }
  if (ACT == kActSilu) return z * sigmoid32(z);
  if (ACT == kActGelu) return z * normal_below(z);
  return z;
}
template <int ACT, bool F32 = false>
__device__ __forceinline__ float act_slope(float z) {
  if (ACT == kActRelu) return z > 0.0f ? 1.0f : z != z ? z : 0.0f;
  if (ACT == kActSilu && F32) {
    const float e = expf(-fabsf(z)), large = 1.0f / (1.0f + e), small = e * large;
    return z < 0.0f ? small * (1.0f + z * large) : large * (1.0f + z * small);
  }
  if (ACT == kActSilu) {
    const float q = sigmoid32(z);
    return q * (1.0f + z * (1.0f - q));
  }
  if (ACT == kActGelu) return fmaf(z * 0.3989422804f, bell(z), normal_below(z));
  return 1.0f;
}
// f(std::integral_constant<int, act>): kernels have the activation as a parameter, since a
// choice at every value costs more than the value (20 us a 256 x 256 tile).
template <class F>
auto with_act(int act, F&& f) {
  switch (act) {
    case kActRelu: return f(std::integral_constant<int, kActRelu>{});
    case kActSilu: return f(std::integral_constant<int, kActSilu>{});
    case kActGelu: return f(std::integral_constant<int, kActGelu>{});
    default: return f(std::integral_constant<int, kActNone>{});
  }
}

// ---------------------------------------------------------------------------
// Operands and epilogue of one product.
// ---------------------------------------------------------------------------
struct LinArgs {
  const void* A;
  const void* B;
  int lda, ldb;          // elements between rows as they lie in memory
  int rows, cols, red;   // C [rows, cols], dense; length of the reduction
  int S;                 // ranges of the reduction; S > 1: sums go to part [S][rows][cols]
  float* part;
  // epilogue
  const float* bias;     // [cols]
  const void* mul;       // [rows, cols]
  const void* res;
  void* z;               // [rows, cols]: the sum with the bias, or null
  void* out;             // of the operands' type, or
  float* out32;          // fp32: the plain sum
  float* row_sums;       // [2 column tiles][rows]: parts of the sums of A's rows (linear_big_kernel)
};

__device__ __forceinline__ void unpack8(uint4 v, float (&f)[8]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    f[2 * q] = __uint_as_float(w[q] << 16);
    f[2 * q + 1] = __uint_as_float(w[q] & 0xffff0000u);
  }
}
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]),
                    pack_bf16x2(f[6], f[7]));
}

// mul's and res' values of eight consecutive columns of a row.
struct Beside {
  uint4 mul, res;
};
__device__ __forceinline__ Beside load_beside(const LinArgs& a, size_t at) {
  Beside b{};
  if (a.mul != nullptr) b.mul = *reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(a.mul) + at);
  if (a.res != nullptr) b.res = *reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(a.res) + at);
  return b;
}

// Eight consecutive columns of a row, from their sums to memory.
struct Bias8 {
  float4 lo, hi;
};
__device__ __forceinline__ Bias8 load_bias(const LinArgs& a, int col) {
  return {*reinterpret_cast<const float4*>(a.bias + col), *reinterpret_cast<const float4*>(a.bias + col + 4)};
}
template <int ACT>
__device__ __forceinline__ void finish8(const LinArgs& a, size_t at, float (&v)[8], const Beside& o, const Bias8& b) {
  if (a.out32 != nullptr) {
    *reinterpret_cast<float4*>(a.out32 + at) = make_float4(v[0], v[1], v[2], v[3]);
    *reinterpret_cast<float4*>(a.out32 + at + 4) = make_float4(v[4], v[5], v[6], v[7]);
    return;
  }
  if (a.bias != nullptr) {
    v[0] += b.lo.x, v[1] += b.lo.y, v[2] += b.lo.z, v[3] += b.lo.w;
    v[4] += b.hi.x, v[5] += b.hi.y, v[6] += b.hi.z, v[7] += b.hi.w;
  }
  if (a.z != nullptr) *reinterpret_cast<uint4*>(static_cast<bf16_t*>(a.z) + at) = pack8(v);
#pragma unroll
  for (int q = 0; q < 8; ++q) v[q] = act_value<ACT>(v[q]);
  float f[8];
  if (a.mul != nullptr) {
    unpack8(o.mul, f);
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] *= f[q];
  }
  if (a.res != nullptr) {
    unpack8(o.res, f);
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] += f[q];
  }
  *reinterpret_cast<uint4*>(static_cast<bf16_t*>(a.out) + at) = pack8(v);
}

// ---------------------------------------------------------------------------
// A panel: R rows (of C, or columns) by a chunk of 64 of the reduction, in LDS.
// Plain: R rows of 128 bytes, swizzled as in the grouped GEMMs (swz_chunk). Transposed:
// 64 rows (of the reduction) of 2 R bytes, whose 16-byte pieces are swizzled so that the
// four rows of a transposing read lie in different banks. R = 64 or 128.
// ---------------------------------------------------------------------------
constexpr int kChunk = 64;

template <int R>
__device__ __forceinline__ int tr_piece(int row, int piece) {
  return R == 128 ? piece ^ ((row & 3) << 2) : piece ^ (((row >> 1) & 1) << 2);
}

template <int R, bool TR, int W>
struct Panel {
  static_assert(R == 64 || R == 128, "panel rows");
  static constexpr int BYTES = R * kChunk * 2;
  static constexpr int LOADS = BYTES / (1024 * W);
  static constexpr int RB = TR ? 2 * R : 128, PP = RB / 16, RPI = 1024 / RB;
  static_assert(BYTES % (1024 * W) == 0, "loads of a wave");
  const char* base;
  size_t step;  // bytes between chunks
  uint32_t off[LOADS];

  // the panel's first row (column) and how many there are from it on; a load past the
  // last one reads the last, whose results are not stored
  __device__ __forceinline__ void init(const void* p, int ld, int first, int left, int wave, int lane) {
    base = static_cast<const char*>(p) + (TR ? (size_t)first * 2 : (size_t)first * (size_t)ld * 2);
    step = TR ? (size_t)ld * (kChunk * 2) : (size_t)(kChunk * 2);
#pragma unroll
    for (int t = 0; t < LOADS; ++t) {
      const int r = (t * W + wave) * RPI + lane / PP;
      if (TR)
        off[t] = (uint32_t)r * (uint32_t)(ld * 2) + (uint32_t)(min(tr_piece<R>(r, lane % PP) * 8, left - 8) * 2);
      else
        off[t] = (uint32_t)min(r, left - 1) * (uint32_t)(ld * 2) + (uint32_t)(swz_chunk<kChunk>(r, lane % PP) * 16);
    }
  }
  // load t of chunk kc; not live: the operand's first bytes, which are there in any case
  __device__ __forceinline__ void load(int t, int kc, bool live, uint32_t lds, int wave) const {
    const uint32_t msk = live ? 0xffffffffu : 0u;
    dma16a(uniform_ptr(base + (live ? (size_t)kc * step : 0)), off[t] & msk, lds + (uint32_t)((t * W + wave) * 1024));
  }
  // the last, partial chunk (n of 64): through registers, zeros past the end
  __device__ __forceinline__ void load_tail(int kc, int n, u32x4_t (&v)[LOADS], int wave, int lane) const {
    const char* p = base + (size_t)kc * step;
#pragma unroll
    for (int t = 0; t < LOADS; ++t) {
      const int r = (t * W + wave) * RPI + lane / PP;
      const bool in = TR ? r < n : swz_chunk<kChunk>(r, lane % PP) * 8 < n;
      v[t] = in ? *reinterpret_cast<const u32x4_t*>(p + off[t]) : u32x4_t{};
    }
  }
  __device__ __forceinline__ void store_tail(const u32x4_t (&v)[LOADS], char* lds, int wave, int lane) const {
#pragma unroll
    for (int t = 0; t < LOADS; ++t) *reinterpret_cast<u32x4_t*>(lds + (t * W + wave) * 1024 + lane * 16) = v[t];
  }
  // fragment of k-step s for rows [r0, r0 + 32): lane (r = lane % 32, h = lane / 32)
  // holds k = 16 s + 8 h + (0..7) of row r0 + r
  static __device__ __forceinline__ bf16x8_t frag(const char* lds, int r0, int s, int lane) {
    if (!TR) return lds_frag<kChunk>(reinterpret_cast<const bf16_t*>(lds), r0 + (lane & 31), 2 * s + (lane >> 5));
    // a transposing read takes 16 lanes x 8 bytes as 4 rows x 16 columns and hands lane
    // i column i
    const int row = 16 * s + 8 * (lane >> 5) + ((lane & 15) >> 2);
    const int colb = r0 * 2 + 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
    typedef __attribute__((address_space(3))) s16x4_t* lds4;
    const uint32_t at = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds));
    const uint32_t p0 = (uint32_t)(row * RB + tr_piece<R>(row, colb >> 4) * 16 + (colb & 15));
    // (row + 4) & 3 and ((row + 4) >> 1) & 1 are those of row: the same piece, 4 rows on
    const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds4>(at + p0));
    const s16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds4>(at + p0 + 4 * RB));
    struct {
      s16x4_t lo, hi;
    } v = {a, b};
    return __builtin_bit_cast(bf16x8_t, v);
  }
};

// N stripes of a wave's sums, 32 rows x 32 NI columns each, whose lanes hold groups of 4
// consecutive columns of a row, through the wave's own piece of LDS to whole rows of 8
// columns a lane. sums(n, put) puts stripe n's groups: put(row, group of columns, values);
// the stripe's first row and column are r0(n) and c0(n). mul and res are loaded four stripes
// ahead (one ahead, their latencies took 20 us a 256 x 256 tile; the first four before the
// reduction gain nothing on large tiles, 1 % on small ones, and lose 3 % where blocks share a
// CU). Each element is read by the lane that writes it, so out may be one of them. Rows and
// columns past C's are not stored.
template <int ACT, int N, int NI, class Sums, class Row, class Col>
__device__ __forceinline__ void finish_stripes(const LinArgs& a, char* lds, int split, int lane, Sums&& sums, Row&& r0,
                                               Col&& c0) {
  constexpr int RB = NI * 128, PP = RB / 16, IT = PP / 4;
  static_assert(PP == 8 || PP == 16, "row pieces");
  auto key = [](int r) { return PP == 16 ? (r & 15) : ((r >> 1) & 7); };
  asm volatile("" : "+v"(lane));  // what depends on it is computed here, not kept through the K loop
  const int lr = lane / (PP / 2), lc = lane % (PP / 2) * 8;
  const bool biased = a.S == 1 && a.bias != nullptr;
  const bool beside = a.S == 1 && (a.mul != nullptr || a.res != nullptr);
  constexpr int AHEAD = N < 4 ? N : 4;
  Beside o[AHEAD][IT] = {};
  Bias8 b[AHEAD] = {};
  auto row_of = [&](int n, int it) { return r0(n) + it * (128 / PP) + lr; };
  auto in = [&](int n, int it) { return row_of(n, it) < a.rows && c0(n) + lc < a.cols; };
  auto prefetch = [&](int n) {
    if (biased && c0(n) + lc < a.cols) b[n % AHEAD] = load_bias(a, c0(n) + lc);
    if (beside) {
#pragma unroll
      for (int it = 0; it < IT; ++it)
        if (in(n, it)) o[n % AHEAD][it] = load_beside(a, (size_t)row_of(n, it) * (size_t)a.cols + (size_t)(c0(n) + lc));
    }
  };
  auto put = [&](int n) {
    char* buf = lds + (n & 1) * (32 * RB);
    sums(n, [&](int r, int p, f32x4_t v) __attribute__((always_inline)) {
      *reinterpret_cast<f32x4_t*>(buf + r * RB + ((p ^ key(r)) * 16)) = v;
    });
  };
#pragma unroll
  for (int n = 0; n < AHEAD; ++n) prefetch(n);
  put(0);
#pragma unroll
  for (int n = 0; n < N; ++n) {
    // the next stripe goes to LDS while this one's reads return
    const char* buf = lds + (n & 1) * (32 * RB);
    float4 u[IT], w[IT];
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      const int r = it * (128 / PP) + lr, p = lane % (PP / 2);
      u[it] = *reinterpret_cast<const float4*>(buf + r * RB + (((2 * p) ^ key(r)) * 16));
      w[it] = *reinterpret_cast<const float4*>(buf + r * RB + (((2 * p + 1) ^ key(r)) * 16));
    }
    __builtin_amdgcn_sched_barrier(0);
    if (n + 1 < N) put(n + 1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int it = 0; it < IT; ++it) {
      if (in(n, it)) {
        const size_t at = (size_t)row_of(n, it) * (size_t)a.cols + (size_t)(c0(n) + lc);
        float v[8] = {u[it].x, u[it].y, u[it].z, u[it].w, w[it].x, w[it].y, w[it].z, w[it].w};
        if (a.S > 1) {
          float* q = a.part + (size_t)split * (size_t)a.rows * (size_t)a.cols + at;
          *reinterpret_cast<float4*>(q) = u[it];
          *reinterpret_cast<float4*>(q + 4) = w[it];
        } else {
          finish8<ACT>(a, at, v, o[n % AHEAD][it], b[n % AHEAD]);
        }
      }
    }
    if (n + AHEAD < N) prefetch(n + AHEAD);
    __builtin_amdgcn_sched_barrier(0);
  }
}

// Tile of a block: tiles of bands of 8 row tiles, so that what runs together shares
// operands; consecutive tiles to one XCD (block b runs on XCD b % 8).
struct TileAt {
  int mt, nt, split;
};
__device__ __forceinline__ TileAt tile_at(unsigned b, unsigned total, int mts, int nts) {
  const unsigned x = b % 8u, i = b / 8u, q = total / 8u, r = total % 8u;
  const unsigned t = x * q + (x < r ? x : r) + i;
  const unsigned tiles = (unsigned)mts * (unsigned)nts;
  const unsigned split = t / tiles, u = t % tiles;
  const unsigned band = u / (8u * (unsigned)nts), in = u % (8u * (unsigned)nts);
  const unsigned h = min(8u, (unsigned)mts - band * 8u);
  return {(int)(band * 8u + in % h), (int)(in / h), (int)split};
}

// ---------------------------------------------------------------------------
// BM x BN tile, WR x WC waves, NS chunks in LDS by direct loads (pipeline_xk). Bound by its
// fills: 333 x 1336 out of 1000 takes 10.4 us in 126 tiles of 64 x 64, 0.3 us a chunk of 16 KB.
// ---------------------------------------------------------------------------
template <int BM, int BN, int WR, int WC, int NS>
struct TileShape {
  static constexpr int W = WR * WC, WM = BM / WR, WN = BN / WC, MI = WM / 32, NI = WN / 32;
  static constexpr int STAGE = (BM + BN) * kChunk * 2;
  static constexpr int OUT = (MI > 1 ? 2 : 1) * 32 * WN * 4;  // of a wave (finish_stripes)
  static constexpr int LDS = STAGE * NS > W * OUT ? STAGE * NS : W * OUT;
};

template <int BM, int BN, int WR, int WC, int NS, bool TA, bool TB, int ACT>
__device__ __forceinline__ void linear_tile(const LinArgs& a, unsigned block, unsigned blocks, bf16_t* smem) {
  using Sh = TileShape<BM, BN, WR, WC, NS>;
  constexpr int W = Sh::W, WM = Sh::WM, WN = Sh::WN, MI = Sh::MI, NI = Sh::NI;
  using PA = Panel<BM, TA, W>;
  using PB = Panel<BN, TB, W>;
  constexpr int STAGE = Sh::STAGE, OUT = Sh::OUT;
  static_assert(STAGE == PA::BYTES + PB::BYTES, "stage");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave / WC, wn = wave % WC;
  const int mts = (a.rows - 1) / BM + 1, nts = (a.cols - 1) / BN + 1;
  const TileAt at = tile_at(block, blocks, mts, nts);
  const int row0 = uniform_int(at.mt * BM), col0 = uniform_int(at.nt * BN);
  const int chunks = a.red / kChunk;
  const int k0 = uniform_int((int)((long long)at.split * chunks / a.S));
  const int k1 = uniform_int((int)((long long)(at.split + 1) * chunks / a.S));
  PA pa;
  PB pb;
  pa.init(a.A, a.lda, row0, a.rows - row0, wave, lane);
  pb.init(a.B, a.ldb, col0, a.cols - col0, wave, lane);
  // the partial chunk's loads leave first and wait in registers
  const int n = at.split == a.S - 1 ? a.red - chunks * kChunk : 0;
  u32x4_t ta[PA::LOADS] = {}, tb[PB::LOADS] = {};
  if (n > 0) {
    pa.load_tail(chunks, n, ta, wave, lane);
    pb.load_tail(chunks, n, tb, wave, lane);
  }
  f32x16_t acc[MI][NI];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NI; ++j) acc[i][j] = f32x16_t{};
  constexpr int KS = kChunk / 16, LOADS = PA::LOADS + PB::LOADS;
  auto issue = [&](int kc, bool live, bf16_t* st, int part) {
    const uint32_t lds = lds_addr(st);
    auto mine = [&](int t) { return part < 0 || (NS > 2 ? t * KS / LOADS : 0) == part; };
#pragma unroll
    for (int t = 0; t < PA::LOADS; ++t)
      if (mine(t)) pa.load(t, k0 + kc, live, lds, wave);
#pragma unroll
    for (int t = 0; t < PB::LOADS; ++t)
      if (mine(PA::LOADS + t)) pb.load(t, k0 + kc, live, lds + PA::BYTES, wave);
  };
  bf16x8_t fa[2][MI], fb[2][NI];
  auto read = [&](const bf16_t* st, int s, int buf) {
    const char* p = reinterpret_cast<const char*>(st);
#pragma unroll
    for (int i = 0; i < MI; ++i) fa[buf][i] = PA::frag(p, wm * WM + i * 32, s, lane);
#pragma unroll
    for (int j = 0; j < NI; ++j) fb[buf][j] = PB::frag(p + PA::BYTES, wn * WN + j * 32, s, lane);
  };
  auto mma = [&](int s) {
    const int buf = s & 1;
#pragma unroll
    for (int j = 0; j < NI; ++j)
#pragma unroll
      for (int i = 0; i < MI; ++i)
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[buf][j], fa[buf][i], acc[i][j], 0, 0, 0);
  };
  // (the tail's loads are older than the pipeline's, whose waits therefore hold)
  pipeline_xk<NS, LOADS, KS, false, false>(k1 - k0, smem, STAGE / 2, issue, read, mma, [] {});
  if (n > 0) {
    char* p = reinterpret_cast<char*>(smem);
    pa.store_tail(ta, p, wave, lane);
    pb.store_tail(tb, p + PA::BYTES, wave, lane);
    __syncthreads();
    for (int s = 0; s * 16 < n; ++s) {
      read(smem, s, 0);
      mma(0);
    }
    __syncthreads();
  }
  finish_stripes<ACT, MI, NI>(
      a, reinterpret_cast<char*>(smem) + wave * OUT, at.split, lane,
      [&](int n, auto&& put) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            put(lane & 31, j * 8 + 2 * g + (lane >> 5),
                f32x4_t{acc[n][j][4 * g], acc[n][j][4 * g + 1], acc[n][j][4 * g + 2], acc[n][j][4 * g + 3]});
      },
      [&](int n) { return row0 + wm * WM + n * 32; }, [&](int) { return col0 + wn * WN; });
}

template <int BM, int BN, int WR, int WC, int NS, bool TA, bool TB, int ACT>
__global__ __launch_bounds__(WR* WC* kWave) void linear_tile_kernel(LinArgs a) {
  __shared__ __align__(16) bf16_t smem[TileShape<BM, BN, WR, WC, NS>::LDS / 2];
  linear_tile<BM, BN, WR, WC, NS, TA, TB, ACT>(a, blockIdx.x, gridDim.x, smem);
}

// Both products of a gradient in one launch, where neither fills the chip: dx's tiles, then
// dw's.
template <int BM, int BN, int WR, int WC, int NS>
__global__ __launch_bounds__(WR* WC* kWave) void linear_pair_kernel(LinArgs dx, LinArgs dw, unsigned first) {
  __shared__ __align__(16) bf16_t smem[TileShape<BM, BN, WR, WC, NS>::LDS / 2];
  if (blockIdx.x < first)
    linear_tile<BM, BN, WR, WC, NS, false, true, kActNone>(dx, blockIdx.x, first, smem);
  else
    linear_tile<BM, BN, WR, WC, NS, true, true, kActNone>(dw, blockIdx.x - first, gridDim.x - first, smem);
}

// ---------------------------------------------------------------------------
// The 256 x 256 tile: 4 waves (2 x 2), each 128 x 128 as four quadrants (A half, B half)
// of 64 x 64, in phases as the grouped GEMMs' 256-row tile (big_tile): a chunk is four
// 16 KB slots (A0, A1, B0, B1: the halves that every wave's quadrants read), two chunks
// deep; a phase runs one quadrant's 16 MFMAs from registers, reads the fragments of the
// slot that the next phase needs and refills the slot read in the phase before, for the
// chunk after next:
//
//   even chunk  A0 B0 | A0 B1 | A1 B1 | A1 B0     odd chunk  A0 B1 | A0 B0 | A1 B0 | A1 B1
//   reads       B1      A1      A0'     B1'                  B0      A1      A0'     B0'
//
// Either operand may be transposed; its slot is then 64 rows of the reduction by 128 rows
// of C, its fragments two transposing reads each.
//
// 16384 x 2048 out of 7168: 321 us, 1.50 PFLOP/s, with silu and gate 352; 8192 x 2048 out of
// 7168, w transposed, 156 us, 1.54; 7168 x 2048 out of 8192, both transposed, 170 us, 1.42 with
// a tile for 224 of 256 CUs. MFMAs are busy 60 to 72 % of the cycles: the clock, and with it the
// time, is what power leaves; the 16 x 16 x 32 MFMA, its sums in place in the accumulation
// registers, takes a third less of it than the 32 x 32 x 16 (371 -> 349 us with silu and gate).
//
// SUMS: also the sums of A's rows over the reduction (the bias' gradient, where A is dz),
// from the fragments. Column tile j of J takes the chunks j, j + J, ..., a wave one of their
// two k-steps, so a row's sum comes in 2 J parts. A pass over dz for them costs 25 us
// (8192 x 7168).
// ---------------------------------------------------------------------------
constexpr int kSlotBytes = 128 * kChunk * 2;

// Position of a 16-byte piece in a transposed slot's row of 256 bytes. A transposing read has
// its first 32 lanes at rows 0-3 and 8-11 of 32 bytes each: rows r and r + 1 lie 64 bytes
// apart, rows r and r + 8 32, so no two lanes meet in a bank. (Without the latter the LDS
// spent 29 000 of a CU's 312 000 cycles of a dx of 8192 x 7168 x 2048 on conflicts, which its
// MFMAs hid: the time is the same within 0.5 %.)
__device__ __forceinline__ int big_piece(int row, int piece) {
  return piece ^ ((row & 3) << 2) ^ (((row >> 3) & 1) << 1);
}

template <bool TR>
struct BigOperand {
  static constexpr int RB = TR ? 256 : 128, PP = RB / 16, RPI = 1024 / RB;
  const char* base;
  uint64_t step;       // bytes between chunks
  uint32_t off[2][4];  // of load t of half h
  uint64_t next;       // address of the chunk that is loaded next,
  uint32_t records;    // 0 past the last one
  uint32_t fof[2][TR ? 4 : 2];  // fragments in slots of even and odd chunks: 64 KB apart, more than an instruction's offset holds

  // slot row (TR: column) q of half h is the tile's row 128 (q / 64) + 64 h + q % 64
  __device__ __forceinline__ void init(const void* p, int ld, int first, int left, int wsel, int wave, int lane,
                                       uint32_t lds) {
    base = static_cast<const char*>(p) + (TR ? (size_t)first * 2 : (size_t)first * (size_t)ld * 2);
    step = TR ? (uint64_t)ld * (kChunk * 2) : (uint64_t)(kChunk * 2);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int r = (t * 4 + wave) * RPI + lane / PP;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (TR) {
          const int piece = big_piece(r, lane % PP);
          off[h][t] = (uint32_t)r * (uint32_t)(ld * 2) +
                      (uint32_t)(min((piece >> 3) * 128 + h * 64 + (piece & 7) * 8, left - 8) * 2);
        } else {
          off[h][t] = (uint32_t)min((r >> 6) * 128 + h * 64 + (r & 63), left - 1) * (uint32_t)(ld * 2) +
                      (uint32_t)(swz_chunk<kChunk>(r, lane % PP) * 16);
        }
      }
    }
    // lane (r = lane % 16, g = lane / 16) holds k = 32 s + 8 g + (0..7) of row r
    const int g = lane >> 4, r = lane & 15;
    if (TR) {
      const int row = 8 * g + (r >> 2);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int colb = (wsel * 64 + i * 16) * 2 + 8 * (lane & 3);
        fof[0][i] = lds + (uint32_t)(row * RB + big_piece(row, colb >> 4) * 16 + (colb & 15));
        fof[1][i] = fof[0][i] + 4 * kSlotBytes;
        asm("" : "+v"(fof[1][i]));  // a register of its own, not an addition at each read
      }
    } else {
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        fof[0][s] = lds + (uint32_t)((wsel * 64 + r) * RB + swz_chunk<kChunk>(r, 4 * s + g) * 16);
        fof[1][s] = fof[0][s] + 4 * kSlotBytes;
        asm("" : "+v"(fof[1][s]));
      }
    }
  }
  // Chunk kc is next; live: -1, or 0 past the last one. Offsets are in the operand by
  // construction; without records a load brings zeros and reads nothing.
  __device__ __forceinline__ void start(int kc, int live) {
    next = reinterpret_cast<uint64_t>(uniform_ptr(base + (uint64_t)kc * step));
    records = (uint32_t)live;
  }
  __device__ __forceinline__ void advance(int live) {
    next += step;
    records = (uint32_t)live;
  }
  // Load t of half h to the LDS byte address that M0 holds (aim_m0). Between that write of
  // M0 and the load there must be another instruction.
  __device__ __forceinline__ void load(int h, int t) const {
    const u32x4_t srd = {(uint32_t)next, (uint32_t)(next >> 32), records, 0x00020000u};
    asm volatile("buffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(off[h][t]), "s"(srd) : "memory");
  }
  // The same, with the wait states that M0 (one) and a descriptor that vector instructions
  // have written (five: as start leaves it) need and the compiler, not seeing the load,
  // would not keep.
  __device__ __forceinline__ void load_first(int h, int t, uint32_t lds, int at) const {
    const u32x4_t srd = {(uint32_t)next, (uint32_t)(next >> 32), records, 0x00020000u};
    asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 4\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
                 :
                 : "v"(off[h][t]), "s"(srd), "s"(lds), "is"(at)
                 : "memory", "scc");
  }
  // fragment of block i (16 rows of the wave's 64) at k-step s (32 of the chunk's 64) of
  // slot w of a chunk of parity par
  __device__ __forceinline__ bf16x8_t frag(int w, int par, int i, int s) const {
    if constexpr (TR) {
      typedef __attribute__((address_space(3))) s16x4_t* lds4;
      const uint32_t at = fof[par][i] + (uint32_t)(w * kSlotBytes + s * 32 * RB);
      const s16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds4>(at));
      const s16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds4>(at + 4 * RB));
      struct {
        s16x4_t lo, hi;
      } v = {a, b};
      return __builtin_bit_cast(bf16x8_t, v);
    } else {
      typedef __attribute__((address_space(3))) u32x4_t* lds16;
      // rows 16 apart swizzle alike
      return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<lds16>(fof[par][s] + (uint32_t)(w * kSlotBytes + i * 16 * RB)));
    }
  }
  // the partial chunk kc (n of 64) into the slots at `slot` of half h, zeros past its end
  __device__ __forceinline__ void load_tail(int kc, int n, char* lds, int h, int wave, int lane) const {
    const char* p = base + (size_t)kc * step;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int r = (t * 4 + wave) * RPI + lane / PP;
      const bool in = TR ? r < n : swz_chunk<kChunk>(r, lane % PP) * 8 < n;
      uint4 v = make_uint4(0, 0, 0, 0);
      if (in) v = *reinterpret_cast<const uint4*>(p + off[h][t]);
      *reinterpret_cast<uint4*>(lds + (t * 4 + wave) * 1024 + lane * 16) = v;
    }
  }
};

template <bool TA, bool TB, int ACT, bool SUMS>
__global__ __launch_bounds__(256) void linear_big_kernel(LinArgs a) {
  __shared__ __align__(16) bf16_t smem[8 * kSlotBytes / 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  const int mts = (a.rows - 1) / 256 + 1, nts = (a.cols - 1) / 256 + 1;
  const TileAt at = tile_at(blockIdx.x, gridDim.x, mts, nts);
  const int row0 = uniform_int(at.mt * 256), col0 = uniform_int(at.nt * 256);
  const int chunks = a.red / kChunk;
  const int kc0 = uniform_int((int)((long long)at.split * chunks / a.S));
  const int nK = uniform_int((int)((long long)(at.split + 1) * chunks / a.S)) - kc0;
  BigOperand<TA> A;
  BigOperand<TB> B;
  const uint32_t lds = lds_addr(smem), lds0 = lds + wave * 1024;
  A.init(a.A, a.lda, row0, a.rows - row0, wm, wave, lane, lds);
  B.init(a.B, a.ldb, col0, a.cols - col0, wn, wave, lane, lds);
  bf16x8_t fr[4][4][2];  // [slot: A0, A1, B0, B1][block][k-step]
  f32x4_t acc[2][2][4][4];  // [A half][B half][row block][column block]
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[h][b][i][j] = f32x4_t{};
  // load t of slot w of the chunk (of parity par) that its operand is at
  auto issue = [&](int w, int par, int t) __attribute__((always_inline)) {
    w < 2 ? A.load(w & 1, t) : B.load(w & 1, t);
  };
  // M0: the LDS address of that load; nothing else in the loop uses it
  auto aim = [&](int w, int par, int t) __attribute__((always_inline)) {
    asm volatile("s_add_u32 m0, %0, %1" ::"s"(lds0), "is"((par * 4 + w) * kSlotBytes + t * 4096) : "memory", "scc");
  };
  auto issue_slot = [&](int w, int par) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int at = (par * 4 + w) * kSlotBytes + t * 4096;
      w < 2 ? A.load_first(w & 1, t, lds0, at) : B.load_first(w & 1, t, lds0, at);
    }
  };
  auto readf = [&](int w, int par, int i, int q) __attribute__((always_inline)) {
    fr[w][i][q] = w < 2 ? A.frag(w, par, i, q) : B.frag(w, par, i, q);
  };
  // As inline assembly, in place in the accumulation registers: as a builtin the compiler
  // gives result and addend of these small blocks different registers and moves them about.
  // It does not see that this is an MFMA: its sums are read by other instructions only
  // after the wait that follows the last one (settle).
  auto mma = [&](int ha, int hb, int i, int j, int q) __attribute__((always_inline)) {
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0"
                 : "+a"(acc[ha][hb][i][j])
                 : "v"(fr[2 + hb][j][q]), "v"(fr[ha][i][q]));
  };
  // One phase: the MFMAs of quadrant (ha, hb); reads slot rw (of parity rp), refills slot iw
  // (of parity ip; its last read was the phase before). step(): what moves a descriptor on.
  // In exactly this order: an MFMA takes 16 cycles of the matrix pipe and 4 of the wave's
  // issue, so the gap after it holds two or three other instructions; more would leave the
  // pipe idle.
  auto phase = [&](int ha, int hb, int rw, int rp, int iw, int ip, auto&& step) __attribute__((always_inline)) {
    wait_lgkmcnt0();      // the fragments read in the last phase are here
    wait_vmcnt<6 * 4>();  // this wave's loads of slot rw landed
    lds_barrier();        // everyone's; and everyone has read slot iw
#pragma unroll
    for (int g = 0; g < 32; ++g) {
      __builtin_amdgcn_sched_barrier(0);
      mma(ha, hb, (g >> 2) & 3, g & 3, g >> 4);
      __builtin_amdgcn_sched_barrier(0);
      if (g < 16 && g % 2 == 1) readf(rw, rp, (g >> 1) & 3, g >> 3);
      if (g == 0) step();
      if (g % 8 == 2) aim(iw, ip, g >> 3);
      if (g % 8 == 4) issue(iw, ip, g >> 3);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto keep = [] {};
  float sum[2][4] = {};  // [A half][row block]: of this lane's row, its part of the reduction
  int sum_at = at.nt;  // the next chunk whose rows this block sums
  auto add_rows = [&](int h, int s) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // said differently for either k-step: merged into one piece of code, the choice
      // would index the fragments, which then were in memory
      u32x4_t q = __builtin_bit_cast(u32x4_t, fr[h][i][s]);
      if (s == 0)
        asm volatile("; k-step 0" : "+v"(q));
      else
        asm volatile("; k-step 1" : "+v"(q));
      float f[8];
      unpack8(__builtin_bit_cast(uint4, q), f);
      sum[h][i] += ((f[0] + f[1]) + (f[2] + f[3])) + ((f[4] + f[5]) + (f[6] + f[7]));
    }
  };
  auto sums_of = [&]([[maybe_unused]] int h, [[maybe_unused]] int c) __attribute__((always_inline)) {
    if constexpr (SUMS) {
      if (c == sum_at) {
        if (wn == 0)
          add_rows(h, 0);
        else
          add_rows(h, 1);
        if (h == 1) sum_at += nts;
      }
    }
  };
  // -1 if there is a chunk c, else 0: in scalar registers, where a comparison would be
  // widened in vector registers
  auto live = [&](int c) __attribute__((always_inline)) {
    int v;
    asm("s_cmp_lt_i32 %1, %2\n\ts_cselect_b32 %0, -1, 0" : "=s"(v) : "s"(c), "s"(nK) : "scc");
    return v;
  };
  // wait states between an MFMA and other readers of its result (at most 11 of 4 passes)
  auto settle = [&]() __attribute__((always_inline)) { asm volatile("s_nop 15\n\ts_nop 7" ::: "memory"); };
  if (nK > 0) {
    A.start(kc0, -1);
    B.start(kc0, -1);
    // slots in the order they are read, nine of them
    issue_slot(0, 0);
    issue_slot(2, 0);
    issue_slot(3, 0);
    issue_slot(1, 0);
    A.advance(live(1));
    B.advance(live(1));
    issue_slot(0, 1);
    issue_slot(3, 1);
    issue_slot(2, 1);
    issue_slot(1, 1);
    A.advance(live(2));
    wait_vmcnt<6 * 4>();  // A0, B0 of chunk 0
    lds_barrier();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        readf(0, 0, i, q);
        readf(2, 0, i, q);
      }
    wait_lgkmcnt0();
    lds_barrier();  // every wave has read A0 of chunk 0
    issue_slot(0, 0);
    // a chunk's four phases: its last one loads A0 of the chunk after the one that the
    // others load
    auto even = [&](int c) __attribute__((always_inline)) {
      phase(0, 0, 3, 0, 2, 0, [&]() __attribute__((always_inline)) { B.advance(live(c + 2)); });
      phase(0, 1, 1, 0, 3, 0, keep);
      sums_of(0, c);
      phase(1, 1, 0, 1, 1, 0, keep);
      phase(1, 0, 3, 1, 0, 1, [&]() __attribute__((always_inline)) { A.advance(live(c + 3)); });
      sums_of(1, c);
    };
    int c = 0;
    for (; c + 1 < nK; c += 2) {
      even(c);
      phase(0, 1, 2, 1, 3, 1, [&]() __attribute__((always_inline)) { B.advance(live(c + 3)); });
      phase(0, 0, 1, 1, 2, 1, keep);
      sums_of(0, c + 1);
      phase(1, 0, 0, 0, 1, 1, keep);
      phase(1, 1, 2, 0, 0, 0, [&]() __attribute__((always_inline)) { A.advance(live(c + 4)); });
      sums_of(1, c + 1);
    }
    if (c < nK) even(c);
    wait_lgkmcnt0();
    wait_vmcnt<0>();
    lds_barrier();  // no load is in flight and every wave is done with the slots
  }
  const int n = a.red - chunks * kChunk;
  if (n > 0 && at.split == a.S - 1) {
    char* p = reinterpret_cast<char*>(smem);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      A.load_tail(chunks, n, p + h * kSlotBytes, h, wave, lane);
      B.load_tail(chunks, n, p + (2 + h) * kSlotBytes, h, wave, lane);
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      if (q * 32 < n) {
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
          for (int i = 0; i < 4; ++i) readf(w, 0, i, q);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int j = 0; j < 4; ++j) mma(h, b, i, j, q);
        if (SUMS && at.nt == 0 && wn == q) {
          if (q == 0)
            add_rows(0, 0), add_rows(1, 0);
          else
            add_rows(0, 1), add_rows(1, 1);
        }
      }
    }
    __syncthreads();
  }
  settle();
  if (SUMS) {
    // the four lanes of a row hold parts of it
    float* p = a.row_sums + (size_t)(2 * at.nt + wn) * (size_t)a.rows;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = row0 + wm * 128 + h * 64 + i * 16 + (lane & 15);
        float v = sum[h][i];
        v += __shfl_xor(v, 16, kWave);
        v += __shfl_xor(v, 32, kWave);
        if (lane < 16 && row < a.rows) p[row] = v;
      }
  }
  // stripe n: B half n / 4, A half n / 2 % 2, row blocks 2 (n % 2) and the next
  finish_stripes<ACT, 8, 2>(
      a, reinterpret_cast<char*>(smem) + wave * 16384, at.split, lane,
      [&](int n, auto&& put) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            put(16 * i + (lane & 15), 4 * j + (lane >> 4), acc[(n >> 1) & 1][n >> 2][2 * (n & 1) + i][j]);
      },
      [&](int n) { return row0 + wm * 128 + (n & 3) * 32; }, [&](int n) { return col0 + wn * 128 + (n >> 2) * 64; });
}

// ---------------------------------------------------------------------------
// Few rows (of x): 16 MB of them by C columns a block. The weights are read once, from
// memory to the 16 x 16 x 32 MFMA's registers, the reduction dealt to the W waves k-step
// by k-step; their sums are joined in LDS. With one row it is a chain of three latencies
// (operands, join, stores) around the weights' bytes. All loads of G k-steps are in flight
// together; a second set of registers, so that they never run dry, gained nothing.
//
// C = 8, for at most 8 rows: the MFMA's 16 columns are those 8 over two halves of a k-step of
// 64, its 16 rows the 8 over the same halves; the two of the four products whose halves agree
// are added. A load then takes whole lines, and there are twice the blocks. Taken up to 5120
// columns on 256 CUs, whatever the reduction (us, 16 columns / 8; one row: 2048 out of 8192 12.8 /
// 8.6, 4096 16.7 / 13.9, 5120 25.6 / 18.1, 4.6 TB/s, 2048 out of 2048 4.6 / 4.1; 8 rows: 2048 out of
// 8192 16.3 / 11.2, 5120 out of 2048 9.0 / 10.0). Beyond, it loses with short reductions (7168 out
// of 2048 8.0 / 8.8, 14336 13.1 / 15.2) and would win with long ones of one row (7168 out of 8192
// 27.5 / 23.5, 14336 49.8 / 41.3).
// ---------------------------------------------------------------------------
template <int MB, int C, int W, int G, int ACT>
__global__ __launch_bounds__(W* kWave) void linear_few_kernel(LinArgs a) {
  static_assert(C == 16 || (C == 8 && MB == 1), "columns of a block");
  constexpr int KW = C == 16 ? 32 : 64, PER = C == 16 ? 2 : 1;  // k of a step; lanes of a row of the epilogue
  __shared__ __align__(16) float part[W][MB][16][16];  // [wave][..][row][column]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r = lane & (C - 1), rr = lane & 15, g = lane >> 4;
  const int col0 = (int)blockIdx.x * C;
  // what the epilogue needs, by the lanes that run it
  const int er = tid / PER, ec = col0 + tid % PER * 8;
  const bool mine = tid < MB * C * PER && er < a.rows && ec < a.cols;
  const size_t at = (size_t)er * (size_t)a.cols + (size_t)ec;
  Beside o{};
  Bias8 b{};
  if (mine) {
    o = load_beside(a, at);
    if (a.bias != nullptr) b = load_bias(a, ec);
  }
  const bf16_t* w = static_cast<const bf16_t*>(a.B) + (size_t)min(col0 + r, a.cols - 1) * (size_t)a.ldb;
  const bf16_t* x[MB];
#pragma unroll
  for (int m = 0; m < MB; ++m) x[m] = static_cast<const bf16_t*>(a.A) + (size_t)min(m * 16 + r, a.rows - 1) * (size_t)a.lda;
  f32x4_t acc[MB];
#pragma unroll
  for (int m = 0; m < MB; ++m) acc[m] = f32x4_t{};
  // the lane's 8 elements of a k-step are there or not (K % 8 == 0)
  const int steps = (a.red + KW - 1) / KW;
  for (int s0 = wave; s0 < steps; s0 += W * G) {
    uint4 fw[G], fx[G][MB];
#pragma unroll
    for (int q = 0; q < G; ++q) {
      const int k = (s0 + q * W) * KW + 8 * g + (C == 8 ? 32 * (rr >> 3) : 0);
      const bool in = k < a.red;
      fw[q] = in ? *reinterpret_cast<const uint4*>(w + k) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int m = 0; m < MB; ++m) fx[q][m] = in ? *reinterpret_cast<const uint4*>(x[m] + k) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int q = 0; q < G; ++q)
#pragma unroll
      for (int m = 0; m < MB; ++m)
        acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(fw[q]), as_bf16x8(fx[q][m]), acc[m], 0, 0, 0);
  }
  // the lane holds columns 4 g .. 4 g + 3 of row rr
#pragma unroll
  for (int m = 0; m < MB; ++m) *reinterpret_cast<f32x4_t*>(&part[wave][m][rr][4 * g]) = acc[m];
  __syncthreads();
  if (!mine) return;
  float v[8] = {};
  auto add = [&](const float* p) {
    const float4 u = *reinterpret_cast<const float4*>(p), y = *reinterpret_cast<const float4*>(p + 4);
    v[0] += u.x, v[1] += u.y, v[2] += u.z, v[3] += u.w, v[4] += y.x, v[5] += y.y, v[6] += y.z, v[7] += y.w;
  };
#pragma unroll
  for (int q = 0; q < W; ++q) {
    add(&part[q][0][er][tid % PER * 8]);
    if (C == 8) add(&part[q][0][8 + er][8]);
  }
  finish8<ACT>(a, at, v, o, b);
}

// Joins the S partial sums of every output, in their order.
template <int ACT>
__global__ __launch_bounds__(256) void linear_join_kernel(LinArgs a) {
  const size_t n8 = (size_t)a.rows * (size_t)(a.cols / 8), plane = (size_t)a.rows * (size_t)a.cols;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n8; i += (size_t)gridDim.x * 256) {
    const float4 u = sum_splits(a.part + i * 8, plane, a.S), w = sum_splits(a.part + i * 8 + 4, plane, a.S);
    float v[8] = {u.x, u.y, u.z, u.w, w.x, w.y, w.z, w.w};
    Bias8 b{};
    if (a.bias != nullptr) b = load_bias(a, (int)(i % (size_t)(a.cols / 8)) * 8);
    finish8<ACT>(a, i * 8, v, load_beside(a, i * 8), b);
  }
}

// ---------------------------------------------------------------------------
// fp32 (the tiny layer, a parity configuration): a 64 x 64 tile, 4 x 4 outputs a
// thread, plain sums.
// ---------------------------------------------------------------------------
template <bool TA, bool TB, int ACT>
__global__ __launch_bounds__(256) void linear_f32_kernel(LinArgs a) {
  __shared__ float la[16][65], lb[16][65];
  const int tid = threadIdx.x, tx = tid % 16, ty = tid / 16;
  const int nts = (a.cols - 1) / 64 + 1;
  const int row0 = (int)(blockIdx.x / (unsigned)nts) * 64, col0 = (int)(blockIdx.x % (unsigned)nts) * 64;
  const float *A = static_cast<const float*>(a.A), *B = static_cast<const float*>(a.B);
  float acc[4][4] = {};
  for (int k0 = 0; k0 < a.red; k0 += 16) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int i = q * 256 + tid;
      const int ra = TA ? i % 64 : i / 16, ka = TA ? i / 64 : i % 16;
      const int rb = TB ? i % 64 : i / 16, kb = TB ? i / 64 : i % 16;
      la[ka][ra] = row0 + ra < a.rows && k0 + ka < a.red
                       ? A[TA ? (size_t)(k0 + ka) * a.lda + row0 + ra : (size_t)(row0 + ra) * a.lda + k0 + ka]
                       : 0.0f;
      lb[kb][rb] = col0 + rb < a.cols && k0 + kb < a.red
                       ? B[TB ? (size_t)(k0 + kb) * a.ldb + col0 + rb : (size_t)(col0 + rb) * a.ldb + k0 + kb]
                       : 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(la[k][ty * 4 + i], lb[k][tx + 16 * j], acc[i][j]);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int row = row0 + ty * 4 + i, col = col0 + tx + 16 * j;
      if (row >= a.rows || col >= a.cols) continue;
      const size_t at = (size_t)row * a.cols + col;
      float v = acc[i][j];
      if (a.bias != nullptr) v += a.bias[col];
      if (a.z != nullptr) static_cast<float*>(a.z)[at] = v;
      v = act_value<ACT, true>(v);
      if (a.mul != nullptr) v *= static_cast<const float*>(a.mul)[at];
      if (a.res != nullptr) v += static_cast<const float*>(a.res)[at];
      (a.out32 != nullptr ? a.out32 : static_cast<float*>(a.out))[at] = v;
    }
}

// ---------------------------------------------------------------------------
// dz = dy * mul * act'(z), dmul = dy * act(z), and partial sums of dz's columns (of the
// fp32 values, before dz is rounded). A block: L lanes of 8 columns by R rows at a time, of
// a range of rows. Whole rows of 512 bytes where there are rows for many ranges (8192 x 7168
// for the bias alone: 19.8 us, 5.9 TB/s; 64 columns by 32 rows 30 us); 64 columns by 128 rows
// and one range, without a join, for few; 32 columns by 256 rows where the matrix is small
// (act_narrow): few blocks, so what counts is how many rows are in flight together.
// ---------------------------------------------------------------------------
struct ActBackwardArgs {
  const void *dy, *z, *mul;
  void *dz, *dmul;  // or null
  float* db;        // [P][cols], or null
  int rows, cols, P;
};

// v plus the value of the lane N places on in the 16-lane row
template <int N>
__device__ __forceinline__ float plus_ror(float v) {
  const int i = __builtin_bit_cast(int, v);
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(i, i, 0x120 | N, 0xf, 0xf, false));
}

template <bool BF16, int ACT, int L, int R>
__global__ __launch_bounds__(L* R) void act_backward_kernel(ActBackwardArgs a) {
  constexpr int PARTS = L < 16 ? L * R / kWave : R;
  __shared__ float sums[PARTS][8 * L];
  const int tid = threadIdx.x, c8 = tid % L, ry = tid / L;
  const int cb = (int)(blockIdx.x / (unsigned)a.P), p = (int)(blockIdx.x % (unsigned)a.P);
  const int col = cb * 8 * L + c8 * 8;
  const int r0 = (int)((long long)p * a.rows / a.P), r1 = (int)((long long)(p + 1) * a.rows / a.P);
  float db[8] = {};
  auto load = [&](const void* q, size_t at, float (&f)[8]) {
    if (BF16) {
      unpack8(*reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(q) + at), f);
    } else {
      const float4 u = *reinterpret_cast<const float4*>(static_cast<const float*>(q) + at);
      const float4 w = *reinterpret_cast<const float4*>(static_cast<const float*>(q) + at + 4);
      f[0] = u.x, f[1] = u.y, f[2] = u.z, f[3] = u.w, f[4] = w.x, f[5] = w.y, f[6] = w.z, f[7] = w.w;
    }
  };
  auto store = [&](void* q, size_t at, const float (&f)[8]) {
    if (BF16) {
      *reinterpret_cast<uint4*>(static_cast<bf16_t*>(q) + at) = pack8(f);
    } else {
      *reinterpret_cast<float4*>(static_cast<float*>(q) + at) = make_float4(f[0], f[1], f[2], f[3]);
      *reinterpret_cast<float4*>(static_cast<float*>(q) + at + 4) = make_float4(f[4], f[5], f[6], f[7]);
    }
  };
  // G rows of a lane at a time, their loads in flight together
  constexpr int G = 2;
  if (col < a.cols) {
    for (int r = r0 + ry; r < r1; r += R * G) {
      float d[G][8] = {}, z[G][8] = {}, m[G][8] = {};
#pragma unroll
      for (int g = 0; g < G; ++g) {
        const size_t at = (size_t)(r + R * g) * (size_t)a.cols + (size_t)col;
        if (r + R * g < r1) {
          load(a.dy, at, d[g]);
          if (a.z != nullptr) load(a.z, at, z[g]);
          if (a.mul != nullptr) load(a.mul, at, m[g]);
        }
      }
#pragma unroll
      for (int g = 0; g < G; ++g) {
        if (r + R * g >= r1) break;
        const size_t at = (size_t)(r + R * g) * (size_t)a.cols + (size_t)col;
        if (a.dmul != nullptr) {
          float f[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) f[q] = d[g][q] * act_value<ACT, !BF16>(z[g][q]);
          store(a.dmul, at, f);
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          if (a.mul != nullptr) d[g][q] *= m[g][q];
          if (ACT != kActNone) d[g][q] *= act_slope<ACT, !BF16>(z[g][q]);
          db[q] += d[g][q];
        }
        if (a.dz != nullptr) store(a.dz, at, d[g]);
      }
    }
  }
  if (a.db == nullptr) return;
  if (L < 16) {  // a wave's rows first
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      if (L == 4) db[q] = plus_ror<4>(db[q]);
      db[q] = plus_ror<8>(db[q]);
      db[q] += __shfl_xor(db[q], 16, kWave);
      db[q] += __shfl_xor(db[q], 32, kWave);
    }
  }
  if (L >= 16 || (tid & 63) < L) {
#pragma unroll
    for (int q = 0; q < 8; ++q) sums[L < 16 ? tid >> 6 : ry][c8 * 8 + q] = db[q];
  }
  __syncthreads();
  if (tid < 8 * L && cb * 8 * L + tid < a.cols) {
    float s = 0.0f;
#pragma unroll
    for (int q = 0; q < PARTS; ++q) s += sums[q][tid];
    a.db[(size_t)p * (size_t)a.cols + cb * 8 * L + tid] = s;
  }
}

// Joins the sums of P ranges, in their order.
__global__ __launch_bounds__(64) void bias_join_kernel(const float* __restrict__ part, int cols, int P,
                                                       float* __restrict__ db) {
  const int c = (int)(blockIdx.x * 64 + threadIdx.x);
  if (c >= cols) return;
  float s = 0.0f;
  for (int p = 0; p < P; p += 16) {  // sixteen loads in flight
    float v[16];
#pragma unroll
    for (int q = 0; q < 16; ++q) v[q] = p + q < P ? part[(size_t)(p + q) * (size_t)cols + c] : 0.0f;
#pragma unroll
    for (int q = 0; q < 16; ++q) s += v[q];
  }
  db[c] = s;
}

__global__ __launch_bounds__(256) void fill_zero_kernel(uint32_t* p, size_t n) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) p[i] = 0;
}

// ---------------------------------------------------------------------------
// Which kernel a product takes.
// ---------------------------------------------------------------------------
struct LinPlan {
  int tile;  // rows and columns of a tile; 0: few rows
  int S;
  int cut;       // the first rows, in whole rounds of large tiles; 0: all rows are alike
  long long ns;  // expected
};
constexpr int kFewRows = 32;

constexpr size_t kLinPartBytes = (size_t)64 << 20;  // partial sums, at most

// few: the kernel of few rows can run (no operand is transposed).
// Few rows: its reads of x grow with the rows, more than 8 of them read the weights in half
// lines, and its blocks go through all of the reduction; tiles do not (us, few rows / tiles:
// 8 rows of 2048 x 7168 10.1 / 17.2, 16 17.7 / 14.8; 16 of 7168 x 2048 11.0 / 13.1; 32 of
// 1024 x 4096 13.3 / 14.1; 12 of 64 x 8192 15.0 / 12.6; 8 of 14336 x 4096 29.8 / 29.0, 1 24.3 /
// 30.6; 32 of 768 x 2048 7.8 / 10.2).
// Tiles: the least time by what a 64-wide chunk of a tile and the rest of the tile took where
// blocks filled the CUs (us; two blocks of a CU together): 256 x 256 1.45 and 9, 128 x 128 0.59
// and 3, two 1.0 and 4.5, 64 x 64 0.30 and 2.5, two 0.41 and 3.5. The reduction may be cut in S
// ranges: a join takes 3.5 us and the partial sums' bytes, written and read, at 4 TB/s.
// (768 x 2048 out of 12265 rows: 64 x 64 tiles uncut 110 us, by this rule 43.)
LinPlan make_plan(int rows, int cols, int red, bool few, long long cus) {
  if (few && rows <= kFewRows && (rows <= 8 || red <= 4096) && (long long)rows * cols * red <= 240000000LL) return {0, 1, 0, 0};
  const long long chunks = red / kChunk, plane = (long long)rows * cols * 4;
  LinPlan best{64, 1, 0, LLONG_MAX};
  for (int t : {256, 128, 64}) {
    const long long n = ((rows - 1LL) / t + 1) * ((cols - 1LL) / t + 1);
    for (int S = 1; S <= 16; ++S) {
      if (S > 1 && (chunks / S < 4 || plane * S > (long long)kLinPartBytes)) break;
      const long long blocks = n * S, c = (chunks + S - 1) / S;
      long long ns;
      if (t == 256)
        ns = ((blocks - 1) / cus + 1) * (c * 1450 + 9000);
      else if (blocks <= cus)
        ns = t == 128 ? c * 590 + 3000 : c * 300 + 2500;
      else
        ns = ((blocks - 1) / (2 * cus) + 1) * (t == 128 ? c * 1000 + 4500 : c * 410 + 3500);
      if (S > 1) ns += 3500 + 2 * S * plane / 4000;
      if (ns < best.ns) best = {t, S, 0, ns};
    }
  }
  // Whole rounds of large tiles and the rest of the rows by a plan of its own, where a last
  // round would leave much of the chip idle (2422 x 14336 x 4096, 560 tiles: 300 -> 262 us). A
  // round that is partly idle runs at a higher clock, so little gains are none (5120 x 8192
  // out of 9000 rows, expected 636 -> 570 us, took 594 -> 621), nor are short reductions.
  const long long nts = (cols - 1LL) / 256 + 1, rounds = (((rows - 1LL) / 256 + 1) * nts) / cus;
  const long long cut = rounds * cus / nts * 256;
  if (cut > 0 && cut < rows && chunks >= 16) {
    const LinPlan rest = make_plan(rows - (int)cut, cols, red, few, cus);
    const long long ns = rounds * (chunks * 1450 + 9000) + rest.ns + 2000;
    if (ns < best.ns * 85 / 100) best = {256, 1, (int)cut, ns};
  }
  return best;
}

// A plan depends on sizes alone; a few are kept, since a call asks for several and making
// one takes a microsecond.
LinPlan linear_plan(int rows, int cols, int red, bool few) {
  struct Kept {
    int rows, cols, red, few;
    long long cus;
    LinPlan plan;
  };
  thread_local Kept kept[64] = {};
  const long long cus = device_cu_count();
  const uint32_t h = ((uint32_t)rows * 2654435761u ^ (uint32_t)cols * 2246822519u ^ (uint32_t)red * 3266489917u ^ (few ? 1u : 0u));
  Kept& k = kept[(h >> 16 ^ h) % 64];
  if (k.rows != rows || k.cols != cols || k.red != red || k.few != (few ? 1 : 0) || k.cus != cus)
    k = {rows, cols, red, few ? 1 : 0, cus, make_plan(rows, cols, red, few, cus)};
  return k.plan;
}

size_t product_ws(int rows, int cols, int red, bool few, bool bf16) {
  if (!bf16 || rows == 0) return 0;
  const LinPlan p = linear_plan(rows, cols, red, few);
  if (p.cut > 0) return product_ws(rows - p.cut, cols, red, few, bf16);
  return p.S > 1 ? (size_t)p.S * (size_t)rows * (size_t)cols * 4 : 0;
}

// The most that product_ws asks for up to these rows, cols and red: of fewer rows a product may be
// cut in more ranges (4096 out of 14336: none for 16384 rows, 64 MB for 1024).
size_t product_ws_up_to(int rows, int cols, int red, bool bf16) {
  const long long ranges = std::min(16, red / kChunk / 4);
  if (!bf16 || ranges < 2) return 0;
  return (size_t)std::min((long long)kLinPartBytes, ranges * rows * cols * 4);
}

template <bool TA, bool TB, int ACT>
hipError_t launch_product(LinArgs a, bool bf16, void* ws, hipStream_t s) {
  if (!bf16) {
    const long long tiles = ((a.rows - 1LL) / 64 + 1) * ((a.cols - 1LL) / 64 + 1);
    linear_f32_kernel<TA, TB, ACT><<<(unsigned)tiles, 256, 0, s>>>(a);
    return hipGetLastError();
  }
  const LinPlan p = linear_plan(a.rows, a.cols, a.red, !TA && !TB);
  if (p.cut > 0) {
    LinArgs top = a;
    top.rows = p.cut, top.S = 1;
    linear_big_kernel<TA, TB, ACT, false><<<(unsigned)(p.cut / 256 * ((a.cols - 1) / 256 + 1)), 256, 0, s>>>(top);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const size_t rows = (size_t)p.cut, out = rows * (size_t)a.cols;
    auto past = [](auto*& q, size_t n) {
      using Q = std::remove_reference_t<decltype(q)>;
      if (q != nullptr) q = (Q)((uintptr_t)q + 2 * n);
    };
    past(a.A, TA ? rows : rows * (size_t)a.lda);
    past(a.mul, out), past(a.res, out), past(a.z, out), past(a.out, out);
    if (a.out32 != nullptr) a.out32 += out;
    a.rows -= p.cut;
    return launch_product<TA, TB, ACT>(a, bf16, ws, s);
  }
  a.S = p.S;
  a.part = static_cast<float*>(ws);
  if constexpr (!TA && !TB) {
    if (p.tile == 0) {
      const unsigned blocks = (unsigned)((a.cols + 15) / 16);
      if (a.rows <= 8 && blocks * 4LL <= device_cu_count() * 5LL)
        linear_few_kernel<1, 8, 8, 8, ACT><<<(unsigned)(a.cols / 8), 512, 0, s>>>(a);
      else if (a.rows <= 16)
        linear_few_kernel<1, 16, 8, 8, ACT><<<blocks, 512, 0, s>>>(a);
      else
        linear_few_kernel<2, 16, 8, 8, ACT><<<blocks, 512, 0, s>>>(a);
      return hipGetLastError();
    }
  }
  const long long tiles = ((a.rows - 1LL) / p.tile + 1) * ((a.cols - 1LL) / p.tile + 1) * p.S;
  if (p.tile == 256) {
    if constexpr (TA && TB) {
      if (a.row_sums != nullptr)
        linear_big_kernel<TA, TB, ACT, true><<<(unsigned)tiles, 256, 0, s>>>(a);
      else
        linear_big_kernel<TA, TB, ACT, false><<<(unsigned)tiles, 256, 0, s>>>(a);
    } else {
      linear_big_kernel<TA, TB, ACT, false><<<(unsigned)tiles, 256, 0, s>>>(a);
    }
  }
  // more blocks than CUs: two to a CU, fewer chunks ahead each (128 x 128, 336 blocks of 64
  // chunks: 70 -> 53 us; 256 blocks, one to a CU in any case, 78 us so, 68 us with four chunks
  // and eight waves)
  else if (p.tile == 128 && tiles <= device_cu_count())
    linear_tile_kernel<128, 128, 2, 4, 4, TA, TB, ACT><<<(unsigned)tiles, 512, 0, s>>>(a);
  else if (p.tile == 128)
    linear_tile_kernel<128, 128, 2, 2, 2, TA, TB, ACT><<<(unsigned)tiles, 256, 0, s>>>(a);
  else if (tiles <= device_cu_count())
    linear_tile_kernel<64, 64, 2, 2, 8, TA, TB, ACT><<<(unsigned)tiles, 256, 0, s>>>(a);
  else
    linear_tile_kernel<64, 64, 2, 2, 4, TA, TB, ACT><<<(unsigned)tiles, 256, 0, s>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.S == 1) return e;
  const size_t n8 = (size_t)a.rows * (size_t)(a.cols / 8);
  linear_join_kernel<ACT><<<(unsigned)std::min<size_t>((n8 + 255) / 256, 8 * (size_t)device_cu_count()), 256, 0, s>>>(a);
  return hipGetLastError();
}

// The activation's gradient by blocks of 32 columns x 256 rows: where they are for half the
// CUs at most and the data are few (us in a captured graph, silu and gate and bias, otherwise /
// so: 333 x 1336 6.5 / 4.8, 1024 x 2048 13.6 / 9.7, 1500 x 4096 24.0 / 19.5, 16384 x 8 32.8 / 7.6; 2048 x 4096 22.9 /
// 24.8, 16384 x 2048 76 / 106: its rows of 64 bytes reach two thirds of the bandwidth), and for
// up to 128 columns, of which the other has lanes to spare (2^20 x 8 236 / 35, x 128 404 / 359).
bool act_narrow(int rows, int cols) {
  return 2 * ((cols - 1) / 32 + 1) <= device_cu_count() && (cols <= 128 || (long long)rows * cols <= (6 << 20));
}

// Row ranges of the bias' sums: one up to 768 or 1024 rows (a join takes 2 us), then 512 rows
// each while blocks of 32 columns fill the chip, or enough blocks of 256 columns for it, at
// least 128 rows each.
int bias_ranges(int rows, int cols) {
  if (act_narrow(rows, cols))
    return rows <= 768 ? 1 : std::min((rows - 1) / 512 + 1, device_cu_count() / ((cols - 1) / 32 + 1));
  if (rows <= 1024) return 1;
  const int cb = (cols - 1) / 256 + 1;
  return std::max(2, std::min((4 * device_cu_count() + cb - 1) / cb, rows / 128));
}

// The most ranges for up to these rows.
int bias_ranges_up_to(int rows, int cols) {
  const int few = (cols - 1) / 32 + 1, cb = (cols - 1) / 256 + 1, cus = device_cu_count();
  int most = rows > 1024 ? std::max(2, std::min((4 * cus + cb - 1) / cb, rows / 128)) : 1;
  if (2 * few <= cus && rows > 768) most = std::max(most, std::min((rows - 1) / 512 + 1, cus / few));
  return most;
}

// Parts of the bias' sums where dw's large tiles make them (0: they do not): dz is dy, and
// the tiles read all of it.
int bias_parts_of_dw(int M, int N, int K, bool bf16) {
  if (!bf16 || M == 0) return 0;
  const LinPlan p = linear_plan(N, K, M, false);
  return p.tile == 256 && p.S == 1 && p.cut == 0 ? 2 * ((K - 1) / 256 + 1) : 0;
}

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace

// Never 0: a call without a workspace asks for its size.
constexpr size_t kLinearWsLeast = 256;

size_t linear_ws_bytes(int M, int N, int K, bool bf16) {
  return std::max(kLinearWsLeast, product_ws_up_to(M, N, K, bf16));
}
size_t linear_ws_needed(int M, int N, int K, bool bf16) {
  return std::max(kLinearWsLeast, product_ws(M, N, K, true, bf16));
}

hipError_t launch_linear(const LinearCall& c, void* ws, hipStream_t s) {
  LinArgs a{};
  a.A = c.x, a.B = c.w, a.lda = c.K, a.ldb = c.ldw;
  a.rows = c.M, a.cols = c.N, a.red = c.K;
  a.bias = c.bias, a.mul = c.mul, a.res = c.residual, a.z = c.z, a.out = c.y;
  return with_act(c.act, [&](auto act) { return launch_product<false, false, decltype(act)::value>(a, c.bf16, ws, s); });
}

size_t linear_backward_ws_bytes(int M, int N, int K, bool bf16) {
  if (M == 0) return kLinearWsLeast;
  // dw's sums have the same size whatever the rows: as many ranges as that allows
  const size_t plane = (size_t)N * (size_t)K * 4;
  const size_t dw = std::min(product_ws_up_to(N, K, M, bf16), kLinPartBytes / plane * plane);
  const int parts = bf16 ? 2 * ((K - 1) / 256 + 1) : 0;
  return align256((size_t)std::max(bias_ranges_up_to(M, N), parts) * (size_t)N * 4) +
         std::max(product_ws_up_to(M, K, N, bf16), dw);
}
size_t linear_backward_ws_needed(int M, int N, int K, bool bf16) {
  if (M == 0) return kLinearWsLeast;
  return align256((size_t)std::max(bias_ranges(M, N), bias_parts_of_dw(M, N, K, bf16)) * (size_t)N * 4) +
         std::max(product_ws(M, K, N, false, bf16), product_ws(N, K, M, false, bf16));
}

hipError_t launch_linear_backward(const LinearBackwardCall& c, void* ws, hipStream_t s) {
  hipError_t e = hipSuccess;
  if (c.M == 0) {
    auto zero = [&](void* p, size_t words) {
      if (p == nullptr || e != hipSuccess) return;
      fill_zero_kernel<<<(unsigned)std::min<size_t>((words + 255) / 256, 2048), 256, 0, s>>>(static_cast<uint32_t*>(p),
                                                                                             words);
      e = hipGetLastError();
    };
    zero(c.dw, (size_t)c.N * c.K / (c.dw_bf16 ? 2 : 1));
    zero(c.dbias, c.N);
    return e;
  }
  const bool own = c.act != kActNone || c.mul != nullptr;  // dz is not dy
  const int parts = bias_parts_of_dw(c.M, c.N, c.K, c.bf16);
  const bool by_dw = parts > 0 && !own && c.dw != nullptr && c.dbias != nullptr;
  const int P = by_dw ? parts : bias_ranges(c.M, c.N);
  auto join_bias = [&] {
    bias_join_kernel<<<(unsigned)((c.N + 63) / 64), 64, 0, s>>>(static_cast<const float*>(ws), c.N, P, c.dbias);
    return hipGetLastError();
  };
  if (own || (c.dbias != nullptr && !by_dw)) {
    ActBackwardArgs b{};
    b.dy = c.dy, b.mul = c.mul, b.dmul = c.dmul;
    b.z = c.act != kActNone || c.dmul != nullptr ? c.z : nullptr;
    b.dz = own ? c.dz : nullptr;
    b.rows = c.M, b.cols = c.N, b.P = P;
    b.db = c.dbias == nullptr ? nullptr : P > 1 ? static_cast<float*>(ws) : c.dbias;
    e = with_act(c.act, [&](auto act) {
      constexpr int A = decltype(act)::value;
      auto go = [&](auto bf16) {
        constexpr bool BF = decltype(bf16)::value;
        if (act_narrow(c.M, c.N))
          act_backward_kernel<BF, A, 4, 256><<<(unsigned)((c.N - 1) / 32 + 1) * (unsigned)P, 1024, 0, s>>>(b);
        else if (P == 1)
          act_backward_kernel<BF, A, 8, 128><<<(unsigned)((c.N - 1) / 64 + 1), 1024, 0, s>>>(b);
        else
          act_backward_kernel<BF, A, 32, 8><<<(unsigned)((c.N - 1) / 256 + 1) * (unsigned)P, 256, 0, s>>>(b);
      };
      c.bf16 ? go(std::true_type{}) : go(std::false_type{});
      return hipGetLastError();
    });
    if (e != hipSuccess) return e;
    if (c.dbias != nullptr && P > 1)
      if ((e = join_bias()) != hipSuccess) return e;
  }
  const void* dz = own ? c.dz : c.dy;
  void* part = static_cast<char*>(ws) + align256((size_t)std::max(P, parts) * (size_t)c.N * 4);
  LinArgs x{}, w{};
  x.A = dz, x.B = c.w, x.lda = c.N, x.ldb = c.ldw;
  x.rows = c.M, x.cols = c.K, x.red = c.N, x.out = c.dx;
  w.A = dz, w.B = c.x, w.lda = c.N, w.ldb = c.K;
  w.rows = c.N, w.cols = c.K, w.red = c.M;
  if (c.dw_bf16)
    w.out = c.dw;
  else
    w.out32 = static_cast<float*>(c.dw);
  if (by_dw) w.row_sums = static_cast<float*>(ws);
  if (c.dx != nullptr && c.dw != nullptr && c.bf16) {
    // In one launch where that is expected to take less than one after the other, with their
    // joins up to four launches, 5 us more than their own times. 64 x 64 tiles: all blocks at once (a
    // chunk takes longer while both reductions run), or those past two a CU after the shorter ones
    // (768 x 2048 out of 333 rows 15.0 -> 10.8 us, 2048 x 768 out of 100 17.1 -> 13.7). 128 x 128
    // tiles: a CU for each (1336 x 1000 out of 1000 rows 24.0 -> 15.9 us, 2048 x 768 out of 1500
    // 25.7 -> 19.8, but out of 700 14.8 -> 19.2; two to a CU took 0.94 to 1.15 of what is done
    // otherwise).
    const LinPlan px = linear_plan(x.rows, x.cols, x.red, false), pw = linear_plan(w.rows, w.cols, w.red, false);
    auto tiles = [](const LinArgs& a, int t) { return ((a.rows - 1LL) / t + 1) * ((a.cols - 1LL) / t + 1); };
    const long long n = tiles(x, 64) + tiles(w, 64), n128 = tiles(x, 128) + tiles(w, 128), slots = 2 * device_cu_count();
    const long long tx = x.red / kChunk * 410LL + 3500, tw = w.red / kChunk * 410LL + 3500;
    const long long cl = std::max(x.red, w.red) / kChunk, cs = std::min(x.red, w.red) / kChunk;
    const long long t64 = n <= slots       ? cl * 300 + cs * 110 + 3500
                          : n <= 2 * slots ? std::max(std::max(tx, tw), std::min(tx, tw) + tw)
                                           : LLONG_MAX;
    const long long t128 = 2 * n128 <= slots ? std::max(x.red, w.red) / kChunk * 590LL + 3000 : LLONG_MAX;
    if (!by_dw && std::min(t64, t128) < px.ns + pw.ns + 5000) {
      x.S = w.S = 1;
      if (t128 < t64)
        linear_pair_kernel<128, 128, 2, 4, 4><<<(unsigned)n128, 512, 0, s>>>(x, w, (unsigned)tiles(x, 128));
      else
        linear_pair_kernel<64, 64, 2, 2, 4><<<(unsigned)n, 256, 0, s>>>(x, w, (unsigned)tiles(x, 64));
      return hipGetLastError();
    }
  }
  if (c.dx != nullptr)
    if ((e = launch_product<false, true, kActNone>(x, c.bf16, part, s)) != hipSuccess) return e;
  if (c.dw != nullptr)
    if ((e = launch_product<true, true, kActNone>(w, c.bf16, part, s)) != hipSuccess) return e;
  if (by_dw) e = join_bias();
  return e;
}

}  // namespace moe
