// Rows in the experts' order, shared by the products grouped by expert.
#pragma once

#include "device_common.hpp"
#include "internal.hpp"

namespace omnimoe {

// Where expert e's positions start, from what the offsets say; past its ends they are not trusted.
__device__ __forceinline__ int within_rows(int o, int M) { return o < 0 ? 0 : o > M ? M : o; }
__device__ __forceinline__ int expert_start(const int32_t* offsets, int e, int M) {
  return offsets ? within_rows(offsets[e], M) : e ? M : 0;
}

// Sum over the lanes up to this one, in the registers' own lanes (no LDS): within rows of sixteen, then over the rows.
__device__ __forceinline__ int wave_incl_scan_dpp(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);  // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);  // row_shr:2
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);  // row_shr:4
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);  // row_shr:8
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);  // row_bcast:15 to rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);  // row_bcast:31 to rows 2 and 3
  return v;
}

struct RowUnit {
  int expert, first, count;  // count <= the unit's most rows
};

// Every expert's positions are cut into units of up to R rows, which are numbered through the experts; returns how many
// there are, and of unit(total) (which may be past the last) what it is. All NT threads of the workgroup take part.
// Up to 256 experts each wave counts by itself, four neighbouring experts a lane; more are spread over the workgroup, whose
// `scratch` (NT / 64 + 4 ints of LDS) is free again after the caller's next barrier.
template <int NT, class Unit>
__device__ __forceinline__ int find_unit(const int32_t* offsets, int N, int M, int R, int* scratch, Unit unit, RowUnit& u) {
  auto units = [&](int lo, int hi) { return hi > lo ? ((unsigned)(hi - lo) + (unsigned)R - 1u) / (unsigned)R : 0u; };
  u = {-1, 0, 0};
  if (!offsets) {
    const int total = (int)units(0, M), want = unit(total);
    if ((unsigned)want < (unsigned)total) u = {0, want * R, M - want * R < R ? M - want * R : R};
    return total;
  }
  if (N <= 256) {
    const int e0 = lane_id() * 4;
    int o[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) o[i] = offsets[e0 + i < N ? e0 + i : N];  // (in flight together)
#pragma unroll
    for (int i = 0; i < 5; ++i) o[i] = within_rows(o[i], M);
    int n[4], mine = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) mine += n[i] = (int)units(o[i], o[i + 1]);
    const int upto = wave_incl_scan_dpp(mine), total = __builtin_amdgcn_readlane(upto, 63), want = unit(total);
    int at = upto - mine;
    const uint64_t has = __ballot(want >= at && want < upto);
    if (!has) return total;
    RowUnit v = {-1, 0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool here = want >= at && want < at + n[i];
      const int first = o[i] + (want - at) * R, left = o[i + 1] - first;
      v.expert = here ? e0 + i : v.expert;
      v.first = here ? first : v.first;
      v.count = here ? (left < R ? left : R) : v.count;
      at += n[i];
    }
    const int lane = __builtin_ctzll(has);
    u = {__builtin_amdgcn_readlane(v.expert, lane), __builtin_amdgcn_readlane(v.first, lane),
         __builtin_amdgcn_readlane(v.count, lane)};
    return total;
  }
  const int tid = threadIdx.x, l = tid & 63, w = tid >> 6;
  const int per = (N + NT - 1) / NT, e0 = tid * per < N ? tid * per : N, e1 = e0 + per < N ? e0 + per : N;
  int mine = 0;
  {
    int lo = expert_start(offsets, e0, M);
    for (int e = e0; e < e1; ++e) {
      const int hi = expert_start(offsets, e + 1, M);
      mine += (int)units(lo, hi);
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
    int lo = expert_start(offsets, e0, M), n = at;
    for (int e = e0; e < e1; ++e) {
      const int hi = expert_start(offsets, e + 1, M), k = (int)units(lo, hi);
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

// t / by for 0 <= t < 2^31 as one multiplication: with 2^(L-1) < by <= 2^L and m = ceil(2^(31+L) / by), which has 32 bits,
// t m / 2^(31+L) exceeds t / by by less than t / 2^31 / by < 1 / by.
struct FastDiv {
  uint32_t m, shift;
  static FastDiv by(uint32_t d) {
    uint32_t l = 0;
    while ((1ull << l) < d) ++l;
    return {(uint32_t)(((1ull << (31 + l)) + d - 1) / d), l};
  }
  __device__ __forceinline__ int operator()(int t) const { return (int)(__umulhi(2u * (uint32_t)t, m) >> shift); }
};

// Where an operand's rows lie: by position, by task or by token. perm is NULL where no operand goes by task.
struct RowOrder {
  const int32_t* perm;
  int M, by_position;  // by_position: all bits, or none
  FastDiv div;         // tasks of a row
  static RowOrder make(const int32_t* perm, int M, int order, int hk) {
    return {perm, M, order == 0 ? -1 : 0, FastDiv::by(order == 2 && hk > 0 ? (uint32_t)hk : 1u)};
  }
  __device__ __forceinline__ int task(int p) const { return perm ? perm[p] : p; }
  // Row of position p, whose task is t; -1 where there is no such task.
  __device__ __forceinline__ int of(int p, int t) const {
    const int row = div(t);
    return (unsigned)t < (unsigned)M ? row ^ ((row ^ p) & by_position) : -1;
  }
  __device__ __forceinline__ int operator()(int p) const { return of(p, task(p)); }
};

// `grid` workgroups of kernel(p, more ..), whose number is p.block0 + blockIdx.x: in several launches where one would have 2^32
// threads or more, which the runtime does not start. Each but the last is of a multiple of eight, so that a number still names
// its XCD.
template <class Kernel, class Args, class... More>
hipError_t launch_numbered(Kernel kernel, int64_t grid, int threads, hipStream_t st, Args p, More... more) {
  if (grid > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
  const int64_t most = (int64_t)(0xFFFFFFFFu / (unsigned)threads) & ~(int64_t)7;
  for (int64_t at = 0; at < grid; at += most) {
    p.block0 = (unsigned)at;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(grid - at < most ? grid - at : most)), dim3(threads), 0, st, p, more...);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  return hipSuccess;
}

}  // namespace omnimoe
