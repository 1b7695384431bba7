// The sum of a 256 x 256 tile by eight waves in two groups that take turns: while the four waves of one group, one on each
// SIMD, keep the matrix cores busy, the other four read their operands from LDS and request copies. tile_sum's waves all do
// both at once; where a tile's copies come from beyond the L2 they then wait for them together.
//
// A stage (64 values of k) is two turns of a group: operand b's rows are cut into two parts of 128, so that the first turn
// takes all of a and part 0 (sixteen reads a wave), the second part 1 (eight), and each has sixteen products a wave. In
// phases of one turn's products, with group 1 a phase behind:
//   phase 4s      group 0 reads a, b0 of stage s; requests b1 of s + 1       group 1: second products of s - 1
//   phase 4s + 1  group 0: first products of s                               group 1 reads a, b0 of s; requests b1 of s + 1
//   phase 4s + 2  group 0 reads b1 of s; requests a, b0 of s + 2             group 1: first products of s
//   phase 4s + 3  group 0: second products of s                              group 1 reads b1 of s; requests a, b0 of s + 2
// Two buffers of each. A request goes into a buffer that both groups have read to the end of (their reads are waited for before
// the barrier between two phases), and is first read five or six phases later; then a wave's eight youngest copies (six of a
// and b0, two of b1) may still be on their way: s_waitcnt vmcnt(8), before the barrier that precedes group 0's reads.
#pragma once

#include "tile_gemm.hpp"

namespace omnimoe {


// Row of the whole tile that row r of part `part` of operand b is: a group's 128 rows of the tile in two halves.
__device__ __forceinline__ int turn_row(int part, int r) { return (r >> 6) * 128 + part * 64 + (r & 63); }

// acc[i][j] += a's rows a0[i] .. + 31 times b's rows: j = 0, 1 rows 64 group + 32 j of part 0, j = 2, 3 the same of part 1.
// OA: 256 rows, OB: 128. K values of k. Every thread of the workgroup takes part; on return the LDS is free.
template <class T, class OA, class OB>
__device__ __forceinline__ void tile_sum_turns(const OA& a, const OB& b0, const OB& b1, int K, const int (&a0)[2], int group,
                                               unsigned char* sa0, unsigned char* sa1, unsigned char* s00, unsigned char* s01,
                                               unsigned char* s10, unsigned char* s11, int wid, int lane,
                                               tg_f32x16 (&acc)[2][4]) {
  static_assert(T::kSize == 2 && OA::kCopies == 4 && OB::kCopies == 2, "eight copies a wave and stage");
  const int n = (K + T::kStep - 1) / T::kStep;
  if (n == 0) return;
  typename T::frag fa[2][4], fb[2][4];
  auto barrier = []() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
  };
  auto wait_reads = []() { __builtin_amdgcn_s_waitcnt(0xC07F); };   // lgkmcnt(0)
  auto wait_copies = []() { __builtin_amdgcn_s_waitcnt(0x0F78); };  // vmcnt(8)
  auto read_a = [&](const unsigned char* st) {
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int i = 0; i < 2; ++i) fa[i][ks] = OA::frag(st, 0, a0[i], ks, lane);
  };
  auto read_b = [&](const unsigned char* st) {
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int j = 0; j < 2; ++j) fb[j][ks] = OB::frag(st, 0, group * 64 + j * 32, ks, lane);
  };
  auto products = [&](auto half) {
    constexpr int kHalf = decltype(half)::value;
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) tile_mma(acc[i][2 * kHalf + j], fa[i][ks], fb[j][ks]);
    __builtin_amdgcn_s_setprio(0);
  };
  auto stage = [&](unsigned char* sa, unsigned char* sb0, unsigned char* sb1, unsigned char* next_b1, int s) {
    read_a(sa);
    read_b(sb0);
    b1.copy(next_b1, 0, 0, s + 1, K, wid, lane);
    wait_reads();
    if (group) wait_copies();
    barrier();
    products(std::integral_constant<int, 0>{});
    if (!group) wait_copies();
    barrier();
    read_b(sb1);
    a.copy(sa, 0, 0, s + 2, K, wid, lane);
    b0.copy(sb0, 0, 0, s + 2, K, wid, lane);
    wait_reads();
    if (group) wait_copies();
    barrier();
    products(std::integral_constant<int, 1>{});
    if (!group) wait_copies();
    barrier();
  };
  a.copy(sa0, 0, 0, 0, K, wid, lane);
  b0.copy(s00, 0, 0, 0, K, wid, lane);
  b1.copy(s10, 0, 0, 0, K, wid, lane);
  a.copy(sa1, 0, 0, 1, K, wid, lane);
  b0.copy(s01, 0, 0, 1, K, wid, lane);
  wait_copies();
  barrier();
  if (group) barrier();  // a phase behind from here on
#pragma unroll 1
  for (int s = 0; s < n; s += 2) {
    stage(sa0, s00, s10, s11, s);
    if (s + 1 < n) stage(sa1, s01, s11, s10, s + 1);
  }
  if (!group) barrier();
  __syncthreads();  // (and the last requests, which nobody reads, have landed)
}

}  // namespace omnimoe
