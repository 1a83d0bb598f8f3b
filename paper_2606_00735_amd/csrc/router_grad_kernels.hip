// Gradient of the router's product z = x W^T + b (gfx950): dx = dz W, dW = dz^T x,
// db = sum_t dz.
//
// dz is fp32, x and W bf16, and the MFMA takes bf16 pairs: dz is split into two
// bf16 terms, hi = bf16(dz) and lo = bf16(dz - hi), each multiplied with the exact
// other operand and summed in fp32. What is dropped is at most 2^-18 of an element
// of dz, 1e-6 of a result's norm. Both reductions run along a dimension that is a row index of
// the bf16 operand (tokens of x, experts of W), so its fragments are read from LDS
// with the transposing read.
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

// Eight fp32 values as hi + lo bf16 fragments.
__device__ __forceinline__ void split8(const float (&f)[8], bf16x8_t& hi, bf16x8_t& lo) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    h[q] = pack_bf16x2(f[2 * q], f[2 * q + 1]);
    l[q] = pack_bf16x2(f[2 * q] - __uint_as_float(h[q] << 16), f[2 * q + 1] - __uint_as_float(h[q] & 0xffff0000u));
  }
  hi = as_bf16x8(make_uint4(h[0], h[1], h[2], h[3]));
  lo = as_bf16x8(make_uint4(l[0], l[1], l[2], l[3]));
}

// ---------------------------------------------------------------------------
// dW and db: a block sums E x 128 columns of x over its range of tokens, 32 at a
// time: the chunk's dz rows (fp32) and x rows (128 columns) go to LDS by direct
// loads, NS stages deep; a wave holds (EP / 2) x 64 of the tile. Each wave splits
// the dz values of its experts as it reads them (lanes across experts: a row of
// LDS is read without conflicts). Experts past E are computed from other rows'
// values and not stored.
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
__global__ __launch_bounds__(256) void router_dw_kernel(RouterGradArgs a) {
  using St = RgStage<EP>;
  constexpr int MI = EP / 64, NJ = 2;  // 32-row blocks of experts, of columns per wave
  __shared__ __align__(16) bf16_t smem[St::BYTES * St::NS / 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = wave >> 1, wn = wave & 1, r32 = lane & 31, h = lane >> 5;
  const int E = a.E, H = a.H;
  const int c0 = (int)blockIdx.x * kRgCols, sp = (int)blockIdx.y;
  const int chunks = (a.T + kRgTok - 1) / kRgTok;
  const int q0 = uniform_int((int)((long long)sp * chunks / a.S));
  const int q1 = uniform_int((int)((long long)(sp + 1) * chunks / a.S));

  // Direct loads. dz: 1 KB of a stage per instruction, 16 bytes a lane (VEC) or 256
  // bytes, 4 a lane; columns past E read the row's last ones. x: 4 rows of 256
  // bytes; columns past H read the row's last ones.
  constexpr int DL = VEC ? 16 : 4, ND = St::DZ / (64 * DL * 4), NX = kRgTok * kRgCols * 2 / 4096;
  constexpr int LOADS = ND + NX;
  auto issue = [&](int q, bool live, bf16_t* st, int) {
    const int t0 = (live ? q0 + q : q1 - 1) * kRgTok;
#pragma unroll
    for (int i = 0; i < ND; ++i) {
      const int byte = ((i * 4 + wave) * 64 + lane) * DL;
      const int row = byte / (EP * 4), e = min((byte % (EP * 4)) / 4, E - DL / 4);
      const int t = min(t0 + row, a.T - 1);
      const float* p = a.dz + (size_t)t * E + e;
      const bf16_t* dst = st + (i * 4 + wave) * 64 * DL / 2;
      if (VEC)
        dma16(p, dst);
      else
        dma4(p, dst);
    }
#pragma unroll
    for (int i = 0; i < NX; ++i) {
      const int row = (i * 4 + wave) * 4 + lane / 16, t = min(t0 + row, a.T - 1);
      const int c = min(c0 + tr_swizzle(row, lane % 16) * 8, H - 8);
      const bf16_t* p = a.x + (size_t)t * H + c;
      dma16(p, st + (St::DZ + (i * 4 + wave) * 1024) / 2);
    }
  };

  f32x16_t acc[1][MI][NJ];
  float db[MI];
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    db[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[0][i][j] = f32x16_t{};
  }
  int q = q0;
  auto compute = [&](bf16_t* st) {
    char* base = reinterpret_cast<char*>(st);
    const int left = a.T - q * kRgTok;  // tokens of this chunk
    if (left < kRgTok) {
      // past the last token: zeros, so that they add nothing
      for (int i = left * EP + threadIdx.x; i < kRgTok * EP; i += 256) reinterpret_cast<float*>(base)[i] = 0.0f;
      for (int i = left * 64 + threadIdx.x; i < kRgTok * 64; i += 256)
        reinterpret_cast<uint32_t*>(base + St::DZ)[i] = 0;
      wait_lgkmcnt0();
      lds_barrier();
    }
    ++q;
    const float* dz = reinterpret_cast<const float*>(base);
#pragma unroll
    for (int s = 0; s < kRgTok / 16; ++s) {
      bf16x8_t xf[NJ];
#pragma unroll
      for (int j = 0; j < NJ; ++j) xf[j] = tr_frag(base + St::DZ, lane, 16 * s, wn * 64 + j * 32);
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        float f[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = dz[(16 * s + 8 * h + k) * EP + wm * (EP / 2) + i * 32 + r32];
        bf16x8_t hi, lo;
        split8(f, hi, lo);
#pragma unroll
        for (int k = 0; k < 8; ++k) db[i] += f[k];
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          acc[0][i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xf[j], hi, acc[0][i][j], 0, 0, 0);
          acc[0][i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(xf[j], lo, acc[0][i][j], 0, 0, 0);
        }
      }
    }
    wait_lgkmcnt0();  // every read of this stage returned before it is refilled
  };
  pipeline<St::NS, LOADS>(
      q1 - q0, smem, St::BYTES / 2, [&](int c, bool live, bf16_t* st) { issue(c, live, st, 0); }, compute);

  if (blockIdx.x == 0 && wn == 0) {
#pragma unroll
    for (int i = 0; i < MI; ++i) {
      const float s = db[i] + __shfl_xor(db[i], 32, kWave);
      const int e = wm * (EP / 2) + i * 32 + r32;
      if (h == 0 && e < E) a.db[(size_t)sp * E + e] = s;
    }
  }
  // rows of the tile are experts; a wave whose 64 columns lie past H stores none
  const int m_end = c0 + wn * 64 < H ? E : 0;
  split_epilogue<MI, NJ, 1, EP / 2, 64>(acc, smem, 0, m_end, 0, H, wm, wn, wave, lane,
                                        a.dw + (size_t)sp * E * H + c0, 0, false);
}

// Sums the S partial sums in order.
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
// dx: a wave keeps the dz rows of its 32 tokens, split, in registers (EP / 16
// fragments of either term) and multiplies them with the columns of W that its
// block walks, 128 at a time; W comes to LDS in pieces of 64 experts x 128 columns
// by direct loads, one stage per piece of a column tile.
// ---------------------------------------------------------------------------
constexpr int kDxRows = 128;

template <int EP, bool VEC>
__global__ __launch_bounds__(256) void router_dx_kernel(RouterGradArgs a, int tiles, int col_split) {
  constexpr int KC = EP / 64;                // pieces of a column tile
  constexpr int NS = KC < 2 ? 2 : KC;        // stages
  constexpr int STAGE = 64 * kRgCols;        // bf16
  constexpr int OUTB = 32 * 128;             // bytes of a wave's output rows, 64 columns at a time
  __shared__ __align__(16) bf16_t smem[NS * STAGE + 4 * OUTB / 2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r32 = lane & 31, h = lane >> 5;
  const int E = a.E, H = a.H;
  const int row0 = (int)blockIdx.x * kDxRows + wave * 32;
  const int tl0 = uniform_int((int)blockIdx.y * tiles / col_split);
  const int tl1 = uniform_int(((int)blockIdx.y + 1) * tiles / col_split);
  bf16x8_t hi[EP / 16], lo[EP / 16];
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
      split8(f, hi[s], lo[s]);
    }
  }
  // piece kc of column tile tl; 16 KB, 4 instructions a wave; rows past E read the last
  const int n = (tl1 - tl0) * KC;
  auto issue = [&](int q, int stage) {
    const int qq = q < n ? q : n - 1;
    const int tl = tl0 + qq / KC, kc = qq % KC;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = (i * 4 + wave) * 4 + lane / 16, e = min(kc * 64 + row, E - 1);
      const int c = min(tl * kRgCols + tr_swizzle(row, lane % 16) * 8, H - 8);
      dma16(a.w + (size_t)e * H + c, smem + stage * STAGE + (i * 4 + wave) * 512);
    }
  };
  wait_vmcnt<0>();
#pragma unroll
  for (int q = 0; q < NS - 1; ++q) issue(q, q);
  char* out = reinterpret_cast<char*>(smem + NS * STAGE) + wave * OUTB;
  for (int tl = tl0; tl < tl1; ++tl) {
    f32x16_t acc[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] = f32x16_t{};
#pragma unroll
    for (int kc = 0; kc < KC; ++kc) {
      const int q = (tl - tl0) * KC + kc;
      const int st = KC < 2 ? q & 1 : kc;
      wait_lgkmcnt0();  // this wave's reads of the piece before returned
      wait_vmcnt<4 * (NS - 2)>();
      lds_barrier();
      issue(q + NS - 1, KC < 2 ? (q + 1) & 1 : (kc + NS - 1) % NS);
      const char* base = reinterpret_cast<const char*>(smem + st * STAGE);
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bf16x8_t wf = tr_frag(base, lane, 16 * s, j * 32);
          acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wf, hi[kc * 4 + s], acc[j], 0, 0, 0);
          acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wf, lo[kc * 4 + s], acc[j], 0, 0, 0);
        }
    }
    // lane (r, h) holds columns 8 g + 4 h + (0..3) of each 32 of its token: to whole
    // rows of 64 columns through the wave's LDS
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
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = i * 8 + lane / 8, p = lane % 8;
        const uint4 v = *reinterpret_cast<const uint4*>(out + at(row, p));
        if (row0 + row < a.T && col < H)
          *reinterpret_cast<uint4*>(a.dx + (size_t)(row0 + row) * H + col + p * 8) = v;
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
  }
  wait_vmcnt<0>();
}

// ---------------------------------------------------------------------------
// fp32 (small layers): plain sums, a thread per output.
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

// thread: (token range sp, expert e, column c); column H is the bias
__global__ __launch_bounds__(256) void router_dw_f32_kernel(const float* __restrict__ dz, const float* __restrict__ x,
                                                            int T, int E, int H, int S, float* __restrict__ dw,
                                                            float* __restrict__ db) {
  const size_t n = (size_t)S * E * (H + 1);
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) {
    const int c = (int)(i % (H + 1)), e = (int)(i / (H + 1) % E), sp = (int)(i / (H + 1) / E);
    const int t0 = (int)((long long)sp * T / S), t1 = (int)((long long)(sp + 1) * T / S);
    float s = 0.0f;
    if (c < H) {
      for (int t = t0; t < t1; ++t) s = fmaf(dz[(size_t)t * E + e], x[(size_t)t * H + c], s);
      dw[((size_t)sp * E + e) * H + c] = s;
    } else {
      for (int t = t0; t < t1; ++t) s += dz[(size_t)t * E + e];
      db[(size_t)sp * E + e] = s;
    }
  }
}

// Token ranges of dW: enough blocks for every CU, at least 64 tokens each.
static int router_ranges(int T, int E, int H, bool bf16) {
  const int cus = device_cu_count();
  const long long blocks = bf16 ? (H + kRgCols - 1) / kRgCols : ((long long)E * (H + 1) + 255) / 256;
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
    router_dw_f32_kernel<<<(unsigned)(((size_t)E * (H + 1) + 255) / 256), 256, 0, s>>>(dz, nullptr, 0, E, H, 1, dw, db);
    return hipGetLastError();
  }
  if (bf16) {
    RouterGradArgs a{dz, static_cast<const bf16_t*>(x), static_cast<const bf16_t*>(w), static_cast<bf16_t*>(dx),
                     pw, pb, T, E, H, S};
    const int tiles = (H + kRgCols - 1) / kRgCols;
    auto run = [&](auto ep, auto vec) {
      constexpr int EP = decltype(ep)::value;
      constexpr bool VEC = decltype(vec)::value;
      router_dw_kernel<EP, VEC><<<dim3((unsigned)tiles, (unsigned)S), 256, 0, s>>>(a);
      e = hipGetLastError();
      if (e != hipSuccess || dx == nullptr) return;
      const int rows = (T + kDxRows - 1) / kDxRows;
      const int split = std::min(tiles, std::max(1, (2 * device_cu_count() + rows - 1) / rows));
      router_dx_kernel<EP, VEC><<<dim3((unsigned)rows, (unsigned)split), 256, 0, s>>>(a, tiles, split);
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
    router_dw_f32_kernel<<<grid((size_t)S * E * (H + 1)), 256, 0, s>>>(dz, static_cast<const float*>(x), T, E, H, S,
                                                                        pw, pb);
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
