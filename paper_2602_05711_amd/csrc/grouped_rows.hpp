// Rows in the experts' order, shared by the products grouped by expert.
#pragma once

#include "device_common.hpp"
#include "internal.hpp"

namespace omnimoe {

// Where expert e's positions start; past its ends the offsets' values are not trusted.
__device__ __forceinline__ int expert_start(const int32_t* offsets, int e, int N, int M) {
  if (!offsets) return e ? M : 0;
  const int o = offsets[e];
  return o < 0 ? 0 : o > M ? M : o;
}

struct RowUnit {
  int expert, first, count;  // count <= the unit's most rows
};

// Every expert's positions are cut into units of up to R rows, which are numbered through the experts; returns how many
// there are, and of unit(total) (which may be past the last) what it is. All NT threads of the workgroup take part: a
// thread counts the units of ceil(N / NT) neighbouring experts. `scratch`: NT / 64 + 4 ints of LDS, free again after the
// caller's next barrier.
template <int NT, class Unit>
__device__ __forceinline__ int find_unit(const int32_t* offsets, int N, int M, int R, int* scratch, Unit unit, RowUnit& u) {
  const int tid = threadIdx.x, l = tid & 63, w = tid >> 6;
  const int per = (N + NT - 1) / NT, e0 = tid * per < N ? tid * per : N, e1 = e0 + per < N ? e0 + per : N;
  int mine = 0;
  {
    int lo = expert_start(offsets, e0, N, M);
    for (int e = e0; e < e1; ++e) {
      const int hi = expert_start(offsets, e + 1, N, M);
      if (hi > lo) mine += (hi - lo + R - 1) / R;
      lo = hi;
    }
  }
  int at = wave_excl_scan_i32(mine);
  if (l == 63) scratch[w] = at + mine;
  if (tid == 0) scratch[NT / 64] = -1;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) {
    const int n = scratch[i];
    if (i < w) at += n;
    total += n;
  }
  const int want = unit(total);
  if (want >= at && want < at + mine) {
    int lo = expert_start(offsets, e0, N, M), n = at;
    for (int e = e0; e < e1; ++e) {
      const int hi = expert_start(offsets, e + 1, N, M), k = hi > lo ? (hi - lo + R - 1) / R : 0;
      if (want < n + k) {
        const int first = lo + (want - n) * R;
        scratch[NT / 64] = e;
        scratch[NT / 64 + 1] = first;
        scratch[NT / 64 + 2] = hi - first < R ? hi - first : R;
        break;
      }
      n += k;
      lo = hi;
    }
  }
  __syncthreads();
  u.expert = __builtin_amdgcn_readfirstlane(scratch[NT / 64]);
  u.first = __builtin_amdgcn_readfirstlane(scratch[NT / 64 + 1]);
  u.count = __builtin_amdgcn_readfirstlane(scratch[NT / 64 + 2]);
  return __builtin_amdgcn_readfirstlane(total);
}

// A position's row: its own number, its task's or its token's; -1 where its task does not exist. perm is NULL where no
// operand goes by task.
__device__ __forceinline__ int row_of(const int32_t* perm, int order, int hk, int M, int p) {
  if (!perm) return p;
  const int t = perm[p];
  if ((unsigned)t >= (unsigned)M) return -1;
  return order == 0 ? p : order == 1 ? t : t / hk;
}

}  // namespace omnimoe
