// The sum of a 256 x 256 tile with tile_gemm.hpp's products and places in LDS and the copies spread over a stage's time.
//
// A stage's copies, all at once behind the barrier, keep the waves from their products for as long as the copies take to be
// issued (64 bytes a cycle: half the time of the stage's products). Here a's are issued among the last quarter's products of
// the stage before the last, b's among the next stage's first, one for every two products; no branch divides these: past
// the sum's end the copies are of zeros. Gate and up projection of 131072 rows, 64 experts, 2048 x 2048: 1041 us where tile_sum's
// loop takes 1080; without SwiGLU, whose accumulators leave it fewer registers, 544 for 65536 rows where tile_sum takes 523.
#pragma once

#include "tile_gemm.hpp"

namespace omnimoe {

// An operand of rows (k contiguous) or columns (MNC) at fixed places of one matrix, TileOperand's without branches.
template <class T, int R, bool MNC, int NW>
struct SpreadOperand : TileOperand<T, R, MNC, NW> {
  typedef TileOperand<T, R, MNC, NW> Tile;
  __device__ __forceinline__ void copy(unsigned char* st, int at, int kt, int K, int wid, int lane) const {
    const char* const from = this->base + kt * this->step;
    const int left = K - kt * T::kStep;
#pragma unroll
    for (int i = 0; i < Tile::kCopies; ++i) {
      const char* p = from + this->off[i];
      p = Tile::chunk_k(i, lane, wid) < left ? p : (const char*)&tile_zeros;
      __builtin_amdgcn_global_load_lds((const void*)p, (tg_lds_ptr)(st + (at + this->lds + i * 1024)), 16, 0, 0);
    }
  }
};

// acc += the sum over K values of k. Waves with work == false (none of their rows of b exists) copy only. ahead(s) runs in
// stage s behind its barrier, before the copies of a's stage s + 2 (for what the operands look up). Every thread of the
// workgroup takes part; on return the LDS is free.
template <class T, class OA, class OB, int MI, int NJ, class Ahead>
__device__ __forceinline__ void spread_sum(const OA& a, const OB& b, int K, const int (&a0)[MI], const int (&b0)[NJ],
                                           bool work, unsigned char* st0, unsigned char* st1, int wid, int lane,
                                           tg_f32x16 (&acc)[MI][NJ], Ahead ahead) {
  if (K <= 0) return;
  const int n = ((K + T::kStep - 1) / T::kStep + 1) & ~1;  // an odd number of stages ends with one of zeros
  auto wait_copies = []() { __builtin_amdgcn_s_waitcnt(0x0F70); };  // vmcnt(0)
  typename T::frag fa[2][MI], fb[2][NJ];
  auto read = [&](const unsigned char* st, int ks) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) fb[ks & 1][j] = OB::frag(st, OA::kBytes, b0[j], ks, lane);
#pragma unroll
    for (int i = 0; i < MI; ++i) fa[ks & 1][i] = OA::frag(st, 0, a0[i], ks, lane);
  };
  auto mma = [&](int ks) {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) tile_mma(acc[i][j], fa[ks & 1][i], fb[ks & 1][j]);
  };
  constexpr int kReads = MI * OA::kReads + NJ * OB::kReads, kMma = MI * NJ * T::kMma;
  constexpr int kPer = (kReads + kMma - 1) / kMma;
  // products of one quarter with the next one's reads, and copies, between them
  auto interleave = [&](auto copies) {
#pragma unroll
    for (int i = 0; i < kMma; ++i) {
      if constexpr (decltype(copies)::value) {
        if (i % 2 == 0) {
          __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);  // VALU
          __builtin_amdgcn_sched_group_barrier(0x010, 1, 0);  // VMEM
        }
      }
      __builtin_amdgcn_sched_group_barrier(0x100, kPer, 0);  // LDS reads
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);     // a product
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto stage = [&](unsigned char* cur, unsigned char* next, int s) {
    __builtin_amdgcn_sched_barrier(0);
    b.copy(next, OA::kBytes, s + 1, K, wid, lane);
    read(cur, 1);
    mma(0);
    interleave(std::true_type{});
    read(cur, 2);
    mma(1);
    interleave(std::false_type{});
    read(cur, 3);
    mma(2);
    interleave(std::false_type{});
    // the wave's copies of stage s + 1 and its reads of stage s are done, and with the barrier everyone's
    wait_copies();
    __syncthreads();
    ahead(s);
    __builtin_amdgcn_sched_barrier(0);
    a.copy(cur, 0, s + 2, K, wid, lane);
    read(next, 0);  // (after the last stage: what is there, unused)
    mma(3);
    interleave(std::true_type{});
  };
  auto idle = [&](unsigned char* cur, unsigned char* next, int s) {
    b.copy(next, OA::kBytes, s + 1, K, wid, lane);
    wait_copies();
    __syncthreads();
    ahead(s);
    a.copy(cur, 0, s + 2, K, wid, lane);
  };
  a.copy(st0, 0, 0, K, wid, lane);
  b.copy(st0, OA::kBytes, 0, K, wid, lane);
  wait_copies();
  __syncthreads();
  a.copy(st1, 0, 1, K, wid, lane);
  if (work) {
    read(st0, 0);
#pragma unroll 1
    for (int s = 0; s < n; s += 2) {
      stage(st0, st1, s);
      stage(st1, st0, s + 1);
    }
  } else {
#pragma unroll 1
    for (int s = 0; s < n; s += 2) {
      idle(st0, st1, s);
      idle(st1, st0, s + 1);
    }
  }
  wait_copies();
  __syncthreads();
}

// The same sum for small tiles, whose stages are shorter than a copy's way: four stages in LDS, three of them on their way.
// Four __shared__ arrays st0 .. st3 hold a stage of both operands each. Every thread of the workgroup takes part; on return the
// LDS is free. 256 rows on a matrix of 2048 x 2048, tiles of 64: 10.6 us, with tile_sum's two stages 18.4; 8192 rows of 16
// experts, tiles of 128: 121 and 175. The weight gradients, whose sums are short and whose rows come from LDS, lost by it (2042
// rows of 16 experts of 512 x 512, both gradients: 16.3 us, dW's stages so too 19.6): fewer workgroups share a compute unit.
template <class T, class OA, class OB, int MI, int NJ>
__device__ __forceinline__ void ring_sum(const OA& a, const OB& b, int K, const int (&a0)[MI], const int (&b0)[NJ],
                                         unsigned char* st0, unsigned char* st1, unsigned char* st2, unsigned char* st3,
                                         int wid, int lane, tg_f32x16 (&acc)[MI][NJ]) {
  if (K <= 0) return;
  const int n = (K + T::kStep - 1) / T::kStep;
  constexpr int kTwo = 2 * (OA::kCopies + OB::kCopies);  // a wave's copies of two stages
  static_assert(kTwo < 64, "vmcnt");
  typename T::frag fa[4][MI], fb[4][NJ];
  auto copy = [&](unsigned char* st, int s) {  // (past the end: zeros, so that the count of copies holds)
    a.copy(st, 0, s, K, wid, lane);
    b.copy(st, OA::kBytes, s, K, wid, lane);
  };
  auto read = [&](const unsigned char* st, int ks) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) fb[ks][j] = OB::frag(st, OA::kBytes, b0[j], ks, lane);
#pragma unroll
    for (int i = 0; i < MI; ++i) fa[ks][i] = OA::frag(st, 0, a0[i], ks, lane);
  };
  auto mma = [&](int ks) {
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) tile_mma(acc[i][j], fa[ks][i], fb[ks][j]);
  };
  auto stage = [&](unsigned char* cur, unsigned char* last, int s) {
    // This stage's copies have arrived, and with the barrier everyone's, and nobody reads the last stage's any more: the wave's
    // reads are back (lgkmcnt), and the compiler moves no access over the empty statements. A fence, which __syncthreads has,
    // would wait for the copies on their way too.
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | (kTwo & 15) | (kTwo >> 4 << 14));  // vmcnt(kTwo) lgkmcnt(0)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    copy(last, s + 3);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) read(cur, ks);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) mma(ks);
    __builtin_amdgcn_sched_barrier(0);
  };
  copy(st0, 0);
  copy(st1, 1);
  copy(st2, 2);
  // (the compiler waits for all copies at a loop's head, whose array it can not tell)
  int s = 0;
#pragma unroll 1
  for (; s + 8 <= n; s += 8) {
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      stage(st0, st3, s + i);
      stage(st1, st0, s + i + 1);
      stage(st2, st1, s + i + 2);
      stage(st3, st2, s + i + 3);
    }
  }
#pragma unroll 1
  for (; s < n; s += 4) {
    stage(st0, st3, s);
    if (s + 1 < n) stage(st1, st0, s + 1);
    if (s + 2 < n) stage(st2, st1, s + 2);
    if (s + 3 < n) stage(st3, st2, s + 3);
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
  __syncthreads();
}

}  // namespace omnimoe
