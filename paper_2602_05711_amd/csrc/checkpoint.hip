// Activation checkpoint in 8 bits: every row of [T, d] in blocks of 32 values, a block held as e4m3 codes times a
// power of two 2^s, s the least exponent (-127 at least) with max |v| <= 448 2^s (448 is e4m3's largest value). The
// scale being a power of two, v 2^-s is exact and the only rounding is that to e4m3 (nearest, ties to even): 2^-4
// relative where |v| >= 2^-6 2^s, 2^-10 2^s absolute below, so at most 2^-4 of a value within 2^14 of its block's
// largest. A block's scale is stored as the byte s + 127. Values that are not finite take no part in the block's maximum
// and are stored as NaN.
// Both ways are bound by memory: each value is read and written once (3.03 bytes a value of bf16). [16384, 2048] bf16:
// 24.2 and 20.1 us, 4.2 and 5.0 TB/s; [509, 2048], which is in the caches: 3.1 us each, a launch's own time.
#include "checkpoint.hpp"
#include "internal.hpp"

namespace omnimoe {
namespace {

// Least s >= -127 with amax <= 448 * 2^s: amax = m 2^k with 1 <= m < 2 and 448 = 1.75 * 2^8, so s = k - 8, one more
// where m > 1.75.
__device__ __forceinline__ int block_exponent(uint32_t amax_bits) {
  if (amax_bits < 0x00800000u) return -127;  // zero, or below 2^-126 = 2 * 2^-127
  const int k = (int)(amax_bits >> 23) - 127;
  const int s = k - 8 + ((amax_bits & 0x007FFFFFu) > 0x00600000u ? 1 : 0);
  return s < -127 ? -127 : s;
}

template <bool BF16>
__device__ __forceinline__ void load8(const void* x, int64_t i, float (&v)[8]) {
  if constexpr (BF16) {
    const uint4 q = *(const uint4*)((const uint16_t*)x + i);
    v[0] = bf16_lo(q.x); v[1] = bf16_hi(q.x); v[2] = bf16_lo(q.y); v[3] = bf16_hi(q.y);
    v[4] = bf16_lo(q.z); v[5] = bf16_hi(q.z); v[6] = bf16_lo(q.w); v[7] = bf16_hi(q.w);
  } else {
    const float4 a = *(const float4*)((const float*)x + i), b = *(const float4*)((const float*)x + i + 4);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
}

// Eight values a thread, four threads a block (the last block of a row may be shorter).
template <bool BF16>
__global__ __launch_bounds__(256) void store_kernel(const void* __restrict__ x, uint8_t* __restrict__ codes,
                                                    uint8_t* __restrict__ scales, int64_t T, int d, int nblk) {
  const int64_t n = T * nblk * 4;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t blk = i >> 2, t = blk / nblk;
    const int b = (int)(blk - t * nblk), c = b * 32 + (int)(i & 3) * 8;
    const bool in = c < d;
    float v[8];
    uint32_t m = 0;
    if (in) {
      load8<BF16>(x, t * d + c, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t a = __float_as_uint(v[e]) & 0x7FFFFFFFu;
        if (a < 0x7F800000u && a > m) m = a;
      }
    }
    // the block's four threads are neighbours and leave the loop together (n is a multiple of 4)
    uint32_t o = (uint32_t)__builtin_amdgcn_update_dpp((int)m, (int)m, 0xB1, 0xF, 0xF, false);
    m = o > m ? o : m;
    o = (uint32_t)__builtin_amdgcn_update_dpp((int)m, (int)m, 0x4E, 0xF, 0xF, false);
    m = o > m ? o : m;
    const int s = block_exponent(m);
    if (!in) continue;
    uint32_t w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float q[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) q[e] = ldexpf(v[4 * h + e], -s);
      int p = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
      w[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], p, true);
#pragma unroll
      for (int e = 0; e < 4; ++e)  // an infinity or NaN: NaN
        if ((__float_as_uint(v[4 * h + e]) & 0x7F800000u) == 0x7F800000u) w[h] |= 0x7Fu << (8 * e);
    }
    *(uint2*)(codes + t * d + c) = make_uint2(w[0], w[1]);
    if ((i & 3) == 0) scales[blk] = (uint8_t)(s + 127);
  }
}

template <bool BF16>
__global__ __launch_bounds__(256) void load_kernel(const uint8_t* __restrict__ codes,
                                                   const uint8_t* __restrict__ scales, void* __restrict__ x,
                                                   int64_t T, int d, int nblk) {
  const int q8 = d / 8;
  const int64_t n = T * q8;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t t = i / q8;
    const int c = (int)(i - t * q8);
    checkpoint_load8<BF16>(codes + i * 8, scales[t * nblk + (c >> 2)], x, i * 8);
  }
}

unsigned grid_of(int64_t threads) {
  const int64_t b = (threads + 255) / 256;
  return (unsigned)(b > 65536 ? 65536 : b);
}

}  // namespace

hipError_t launch_checkpoint_store(int64_t T, int d, bool bf16, const void* x, uint8_t* codes, uint8_t* scales,
                                   hipStream_t st) {
  const int nblk = (d + 31) / 32;
  const unsigned grid = grid_of(T * nblk * 4);
  if (bf16) hipLaunchKernelGGL(store_kernel<true>, dim3(grid), dim3(256), 0, st, x, codes, scales, T, d, nblk);
  else hipLaunchKernelGGL(store_kernel<false>, dim3(grid), dim3(256), 0, st, x, codes, scales, T, d, nblk);
  return hipGetLastError();
}

hipError_t launch_checkpoint_load(int64_t T, int d, bool bf16, const uint8_t* codes, const uint8_t* scales, void* x,
                                  hipStream_t st) {
  const int nblk = (d + 31) / 32;
  const unsigned grid = grid_of(T * (d / 8));
  if (bf16) hipLaunchKernelGGL(load_kernel<true>, dim3(grid), dim3(256), 0, st, codes, scales, x, T, d, nblk);
  else hipLaunchKernelGGL(load_kernel<false>, dim3(grid), dim3(256), 0, st, codes, scales, x, T, d, nblk);
  return hipGetLastError();
}

}  // namespace omnimoe
