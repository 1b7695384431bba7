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

// Two values rounded to bf16, to nearest even, in one instruction (v_cvt_pk_bf16_f32).
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){lo, hi}, bf16x2));
}

// Four neighbouring values, rounded so.
__device__ __forceinline__ void put4(uint16_t* p, float a, float b, float c, float d) {
  *(uint2*)p = make_uint2(bf16_pair(a, b), bf16_pair(c, d));
}
__device__ __forceinline__ void put4(float* p, float a, float b, float c, float d) {
  *(float4*)p = make_float4(a, b, c, d);
}

// silu(g) u for a result in the layer's type, g at least kDeepGate (or NaN): bf16's from the hardware's exp2 and reciprocal,
// whose errors (2^-22 relative, and |g| 2^-23 from the exponent's roundings) are far below its rounding; six instructions instead
// of forty, of which a tile of 256 x 256 has as many as a quarter of its products' time.
template <bool BF16>
__device__ __forceinline__ float swiglu_near(float g, float u) {
  if constexpr (BF16) return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -1.44269504088896341f)) * u;
  else return activation(1, g) * u;
}

// Below, e^-g and its reciprocal leave fp32's normal values (from -87 on) before silu(g) u does. There silu(g) = g e^g to fp32's
// accuracy, formed as g q u q^3 with q = e^(g/4), which is a normal value down to g = -349.
constexpr float kDeepGate = -80.0f;
template <bool BF16>
__device__ __forceinline__ float swiglu(float g, float u) {
  if (!(g < kDeepGate)) return swiglu_near<BF16>(g, u);
  float q;
  if constexpr (BF16) q = __builtin_amdgcn_exp2f(g * (0.25f * 1.44269504088896341f));
  else q = expf(0.25f * g);
  return g * q * u * q * q * q;
}

// (bf16: rounded to nearest even)
template <bool BF16>
__device__ __forceinline__ void store8(void* x, int64_t i, const float (&v)[8]) {
  if constexpr (BF16) {
    *(uint4*)((uint16_t*)x + i) =
        make_uint4(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7]));
  } else {
    *(float4*)((float*)x + i) = make_float4(v[0], v[1], v[2], v[3]);
    *(float4*)((float*)x + i + 4) = make_float4(v[4], v[5], v[6], v[7]);
  }
}

// The same as they lie in memory, for a load that is used later.
template <bool BF16>
struct Raw8 {
  uint4 q[BF16 ? 1 : 2];
  __device__ __forceinline__ void load(const void* x, int64_t i) {
    const uint4* const p = (const uint4*)((const char*)x + i * (BF16 ? 2 : 4));
#pragma unroll
    for (int k = 0; k < (BF16 ? 1 : 2); ++k) q[k] = p[k];
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int k = 0; k < (BF16 ? 1 : 2); ++k) q[k] = make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ void values(float (&v)[8]) const {
    if constexpr (BF16) {
      v[0] = bf16_lo(q[0].x); v[1] = bf16_hi(q[0].x); v[2] = bf16_lo(q[0].y); v[3] = bf16_hi(q[0].y);
      v[4] = bf16_lo(q[0].z); v[5] = bf16_hi(q[0].z); v[6] = bf16_lo(q[0].w); v[7] = bf16_hi(q[0].w);
    } else {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        v[4 * k] = __uint_as_float(q[k].x);
        v[4 * k + 1] = __uint_as_float(q[k].y);
        v[4 * k + 2] = __uint_as_float(q[k].z);
        v[4 * k + 3] = __uint_as_float(q[k].w);
      }
    }
  }
};

}  // namespace omnimoe
