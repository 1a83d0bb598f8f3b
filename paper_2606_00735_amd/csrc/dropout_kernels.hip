// Dropout with a residual, its mask from a counter-based generator and never stored
// (gfx950): out = residual + (u >= threshold ? x * scale : 0).
//
// u of element i is word i % 4 of Philox4x32 with 10 rounds (Salmon, Moraes, Dror, Shaw,
// "Parallel random numbers: as easy as 1, 2, 3", 2011) at counter offset + i / 4 under the
// key `seed`, so a mask depends on the element alone: the gradient's call makes it again,
// whatever the launch.
#include <algorithm>

#include "common.hpp"
#include "launch.hpp"

namespace moe {

namespace {

struct Words {
  uint32_t v[4];
};

__device__ __forceinline__ Words philox(uint64_t counter, uint64_t key) {
  uint32_t a = (uint32_t)counter, b = (uint32_t)(counter >> 32), c = 0, d = 0;
  uint32_t k0 = (uint32_t)key, k1 = (uint32_t)(key >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t u = (uint64_t)a * 0xD2511F53u, v = (uint64_t)c * 0xCD9E8D57u;
    a = (uint32_t)(v >> 32) ^ b ^ k0;
    b = (uint32_t)v;
    c = (uint32_t)(u >> 32) ^ d ^ k1;
    d = (uint32_t)u;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return {{a, b, c, d}};
}

__device__ __forceinline__ float drop(float x, uint32_t u, uint32_t threshold, float scale) {
  return u >= threshold ? x * scale : 0.0f;
}

// Four elements a thread, a counter each; the tail one by one. out may be x or
// residual: a thread reads its elements before it writes them. Bound by memory: 16384 x 7168
// bf16 with a residual, 705 MB, 134.5 us, 5.24 TB/s (a copy of 2 GiB 4.8-5.1); the ten rounds,
// 40 multiplications a counter, hide behind it. fp32 is loaded and stored word by word, which takes
// its toll: the same size, 1.41 GB, 384 us, 3.7 TB/s, without a residual 288 us, 3.3 TB/s.
template <bool BF16, bool RES>
__global__ __launch_bounds__(256) void dropout_kernel(const void* x, const void* residual,
                                                      const uint64_t* __restrict__ rng, long long n,
                                                      uint32_t threshold, float scale, void* out) {
  const uint64_t seed = rng[0], offset = rng[1];
  const long long quads = (n + 3) / 4, step = (long long)gridDim.x * 256;
  for (long long q = (long long)blockIdx.x * 256 + threadIdx.x; q < quads; q += step) {
    const Words u = philox(offset + (uint64_t)q, seed);
    float f[4], r[4] = {};
    const bool whole = 4 * q + 4 <= n;
    const int m = whole ? 4 : (int)(n - 4 * q);
    if (BF16) {
      uint16_t h[4] = {}, g[4] = {};
      const bf16_t* px = static_cast<const bf16_t*>(x) + 4 * q;
      const bf16_t* pr = RES ? static_cast<const bf16_t*>(residual) + 4 * q : nullptr;
      if (whole) {
        *reinterpret_cast<uint2*>(h) = *reinterpret_cast<const uint2*>(px);
        if (RES) *reinterpret_cast<uint2*>(g) = *reinterpret_cast<const uint2*>(pr);
      } else {
        for (int i = 0; i < m; ++i) {
          h[i] = px[i];
          if (RES) g[i] = pr[i];
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = bf16_to_f32(h[i]), r[i] = bf16_to_f32(g[i]);
    } else {
      const float* px = static_cast<const float*>(x) + 4 * q;
      const float* pr = RES ? static_cast<const float*>(residual) + 4 * q : nullptr;
      for (int i = 0; i < 4; ++i) {
        f[i] = i < m ? px[i] : 0.0f;
        if (RES) r[i] = i < m ? pr[i] : 0.0f;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[i] = drop(f[i], u.v[i], threshold, scale);
      if (RES) f[i] += r[i];
    }
    if (BF16) {
      bf16_t* po = static_cast<bf16_t*>(out) + 4 * q;
      if (whole) {
        *reinterpret_cast<uint2*>(po) = make_uint2(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]));
      } else {
        for (int i = 0; i < m; ++i) po[i] = f32_to_bf16(f[i]);
      }
    } else {
      float* po = static_cast<float*>(out) + 4 * q;
      for (int i = 0; i < m; ++i) po[i] = f[i];
    }
  }
}

}  // namespace

hipError_t launch_dropout(const void* x, const void* residual, const uint64_t* rng, long long n, uint32_t threshold,
                          float scale, bool bf16, void* out, hipStream_t s) {
  const long long blocks = ((n + 3) / 4 + 255) / 256;
  const dim3 grid((unsigned)std::min(blocks, 16LL * device_cu_count()));
  auto go = [&](auto kernel) { kernel<<<grid, 256, 0, s>>>(x, residual, rng, n, threshold, scale, out); };
  if (bf16)
    residual ? go(dropout_kernel<true, true>) : go(dropout_kernel<true, false>);
  else
    residual ? go(dropout_kernel<false, true>) : go(dropout_kernel<false, false>);
  return hipGetLastError();
}

}  // namespace moe
