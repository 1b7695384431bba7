// Eight neighbouring values of a row in the layer's type.
#pragma once

#include "device_common.hpp"

namespace omnimoe {

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

// (bf16: rounded to nearest even)
template <bool BF16>
__device__ __forceinline__ void store8(void* x, int64_t i, const float (&v)[8]) {
  if constexpr (BF16) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = (uint32_t)bf16_rne(v[2 * e]) | ((uint32_t)bf16_rne(v[2 * e + 1]) << 16);
    *(uint4*)((uint16_t*)x + i) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
    *(float4*)((float*)x + i) = make_float4(v[0], v[1], v[2], v[3]);
    *(float4*)((float*)x + i + 4) = make_float4(v[4], v[5], v[6], v[7]);
  }
}

}  // namespace omnimoe
