// Values of an 8-bit checkpoint (checkpoint.hip).
#pragma once

#include "device_common.hpp"

namespace omnimoe {

// Eight codes of one block to x[at .. at + 8).
template <bool BF16>
__device__ __forceinline__ void checkpoint_load8(const uint8_t* codes, uint8_t scale, void* x, int64_t at) {
  const float kLargest = __uint_as_float(BF16 ? 0x7F7F0000u : 0x7F7FFFFFu);
  const uint2 w = *(const uint2*)codes;
  const int s = (int)scale - 127;
  float v[8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int p = (int)(h ? w.y : w.x);
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(p, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(p, true);
    const float q[4] = {lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float y = ldexpf(q[e], s);
      // a value next to the type's largest may have been rounded up past it
      v[4 * h + e] = fabsf(y) > kLargest ? copysignf(kLargest, y) : y;
    }
  }
  if constexpr (BF16) {
    uint32_t o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = (uint32_t)bf16_rne(v[2 * e]) | ((uint32_t)bf16_rne(v[2 * e + 1]) << 16);
    *(uint4*)((uint16_t*)x + at) = make_uint4(o[0], o[1], o[2], o[3]);
  } else {
    *(float4*)((float*)x + at) = make_float4(v[0], v[1], v[2], v[3]);
    *(float4*)((float*)x + at + 4) = make_float4(v[4], v[5], v[6], v[7]);
  }
}

}  // namespace omnimoe
