// fp32 values as sums of bf16 ones, for products on the matrix cores that keep more than bf16's eight bits.
#pragma once

#include "device_common.hpp"

namespace omnimoe {

// The bits of v's next part, v to the nearest bf16 value; v becomes what that leaves, exactly. A finite v past bf16's
// largest value (by 2^120 at most) has that as its part, so that the parts' sum stays v; a v that is not finite is its
// own part and leaves zero.
__device__ __forceinline__ uint32_t bf16_part(float& v) {
  uint32_t h = bf16_rne(v);
  const bool finite = (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u;
  if (finite && (h & 0x7F80u) == 0x7F80u) --h;
  v = finite ? v - __uint_as_float(h << 16) : 0.0f;
  return h;
}

}  // namespace omnimoe
