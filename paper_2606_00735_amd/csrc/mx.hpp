// OCP Microscaling FP8 (MXFP8) on gfx950: FP8 E4M3 elements (the OCP
// encoding: bias 7, no infinities, largest finite 448) sharing one E8M0
// scale 2^(c - 127) per 32 consecutive elements along the reduction
// dimension. The paper serves its models in FP8 (Table 2a) without naming a
// scaling scheme; MX block scaling is the one gfx950's scaled MFMA consumes
// directly.
//
// Scale layout used by every MX operand here: the four codes of a row's
// 128-element K chunk form one dword (byte b covers elements
// [32 b, 32 b + 32) of the chunk), and dwords are stored chunk-major:
// scales[chunk][row], so one chunk of a tile's rows is contiguous.
#pragma once

#include "common.hpp"

namespace moe {

constexpr int kMxBlock = 32;   // elements per scale code
constexpr int kMxChunk = 128;  // elements per scale dword

typedef int int32x8_t __attribute__((ext_vector_type(8)));

// Scale code of a block whose largest magnitude is amax (finite, >= 0): the
// shared exponent floor(log2 amax) - 8, 8 being the exponent of E4M3's
// largest power of two (so the block's largest element lands in [256, 512)
// before the clamp to 448), biased by 127 and clamped below at code 0. An
// fp32 with biased exponent E has floor(log2) = E - 127, so the code is
// E - 8; zero, denormal and tiny blocks take code 0 (2^-127).
__device__ __forceinline__ uint32_t mx_scale_code(float amax) {
  const int be = static_cast<int>((__float_as_uint(amax) >> 23) & 0xFFu);
  return be > 8 ? static_cast<uint32_t>(be - 8) : 0u;
}

// 2^-(c - 127) for scale code c: an exact power of two, normal for every code
// a finite fp32 block produces (c <= 246).
__device__ __forceinline__ float mx_inv_scale(uint32_t c) { return __uint_as_float((254u - c) << 23); }

// Four values already divided by their block scale, as E4M3 codes packed
// little-endian (v0 in the low byte): clamped to +-448, then rounded to
// nearest even by v_cvt_pk_fp8_f32 (OCP E4M3 on gfx950; the sign of a value
// that rounds to zero is kept).
__device__ __forceinline__ uint32_t e4m3x4(float v0, float v1, float v2, float v3) {
  auto sat = [](float v) { return fminf(fmaxf(v, -448.0f), 448.0f); };
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(sat(v0), sat(v1), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(sat(v2), sat(v3), w, true);
  return static_cast<uint32_t>(w);
}

// ---------------------------------------------------------------------------
// OCP Microscaling FP4 (MXFP4): E2M1 elements (+-0, 0.5, 1, 1.5, 2, 3, 4, 6)
// under the same 32-element E8M0 scales. A row is padded with zero codes to
// whole chunks of 256 elements = 128 bytes (two codes a byte, the even element
// in the low half), so a chunk is the same 128-byte tile row as 64 bf16 or 128
// E4M3 elements.
//
// The scaled MFMA reads 32 consecutive elements of a row from lane (row, h), h
// = 0, 1, for its 64 elements of K, i.e. one block, and that block's code from
// byte s of a scale register of the same lane. The 8 codes of a chunk are kept
// as two dwords, that of h holding block 2 s + h in byte s: a lane's dword then
// serves all four k-steps of a chunk as it is. Dwords are stored chunk-major,
// scales[chunk][row][2], so one chunk of a tile's rows is contiguous.
//
// A block that holds a NaN or an infinity takes scale code 255, E8M0's NaN (and
// zero element codes): the MFMA makes every product with it a NaN, so a bad
// value shows instead of being clamped to a number.
// ---------------------------------------------------------------------------
constexpr int kMx4Chunk = 256;
constexpr uint32_t kMxNan = 255;

// Bytes of a row of K elements: whole chunks.
__host__ __device__ __forceinline__ int mx4_row_bytes(int K) {
  return (K + kMx4Chunk - 1) / kMx4Chunk * (kMx4Chunk / 2);
}

// Scale code of a block from the largest of its elements' fp32 bits without the
// sign (an integer maximum: NaNs and infinities, which have the largest bits,
// are not lost). E2M1's largest power of two is 2^2: floor(log2 amax) - 2, as in
// mx_scale_code.
__device__ __forceinline__ uint32_t mx4_scale_code(uint32_t amax_bits) {
  const int be = static_cast<int>(amax_bits >> 23);
  return be == 255 ? kMxNan : (be > 2 ? static_cast<uint32_t>(be - 2) : 0u);
}

// 2^(c - 127) as fp32 (a NaN for code 255), the scale operand of the conversions.
__device__ __forceinline__ float mx4_scale(uint32_t c) {
  return __uint_as_float(c == 0 ? 0x00400000u : (c == kMxNan ? 0x7fc00000u : c << 23));
}

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// Byte of a chunk's two scale dwords that holds block b (0..7).
__device__ __forceinline__ int mx4_scale_byte(int b) { return (b & 1) * 4 + (b >> 1); }

// Four values over a block's scale as E2M1 codes in the low 16 bits (v0 in bits
// 0-3): v_cvt_scalef32_pk_fp4_f32 divides, rounds to nearest even and clamps to
// +-6.
__device__ __forceinline__ uint32_t e2m1x4(float v0, float v1, float v2, float v3, float scale) {
  uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, v0, v1, scale, 0);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v2, v3, scale, 1);
}

}  // namespace moe
