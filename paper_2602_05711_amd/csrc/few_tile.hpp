// Products of weight rows with a few tokens, bound by reading the weights once (few.hip, adapters.hip).
//
// Few tokens leave the matrix cores idle, so that a tile of sixteen weight rows x sixteen tokens (v_mfma 16x16) costs
// nothing beside the loads, however many of the sixteen there are. A lane reads 32 neighbouring bytes of a row in two
// loads, so that two instructions cover sixteen whole 128-byte lines; the sum runs over k in that permuted order, the
// same for both operands. A workgroup's waves split k and their tiles are added in wave order through LDS.
#pragma once

#include <type_traits>

#include "device_common.hpp"

namespace omnimoe {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// 16 rows x 16 tokens: acc of lane l, register q is row 4 (l / 16) + q, token l % 16.
template <bool BF16>
struct Chunk;  // 16 bytes of a row
template <>
struct Chunk<true> {
  static constexpr int kElems = 8;
  static __device__ __forceinline__ void mma(f32x4& acc, const uint4& a, const uint4& b) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc,
                                                  0, 0, 0);
  }
};
template <>
struct Chunk<false> {
  static constexpr int kElems = 4;
  static __device__ __forceinline__ void mma(f32x4& acc, const uint4& a, const uint4& b) {
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.x), __uint_as_float(b.x), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.y), __uint_as_float(b.y), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.z), __uint_as_float(b.z), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w), __uint_as_float(b.w), acc, 0, 0, 0);
  }
};

// RB x 16 weight rows against NB token operands, summed over this wave's steps (w of W): a step is four lanes x 32 bytes
// (128 bytes of every row), a wave takes U neighbouring ones at a time and has their weights in flight together, U as
// large as leaves every wave some.
// row: this lane's weight row in each of the row blocks, of `chunks` times 16 bytes; tok: this lane's token row in each of
// the operands (lanes past the last token have that one's: their columns of the tile are not used). Operand n has tile
// b NACC + n of row block b; those past the last of the NACC tiles are summed in that one. The loads are unconditional;
// chunks past the row's end read its last one and become zeros, the token's too (its infinity times a weight's zero would
// not be one).
template <bool BF16, int RB, int NB, int NACC, int W, int U>
__device__ __forceinline__ void wave_steps(const uint4* const (&row)[RB], const uint4* const (&tok)[NB], int chunks, int w,
                                           f32x4 (&acc)[RB * NACC]) {
  const int quad = (threadIdx.x & 63) >> 4;
  auto steps = [&](int s0, auto whole) {
    constexpr bool kWhole = decltype(whole)::value;
    auto chunk = [&](int i, int e) {
      const int c = (s0 + i) * 8 + quad * 2 + e;
      return kWhole || c < chunks ? c : chunks - 1;
    };
    uint4 a[U][2][RB];
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int r = 0; r < RB; ++r) a[i][e][r] = row[r][chunk(i, e)];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      uint4 b[2][NB];
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int n = 0; n < NB; ++n) b[e][n] = tok[n][chunk(i, e)];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (!kWhole && (s0 + i) * 8 + quad * 2 + e >= chunks) {
#pragma unroll
          for (int r = 0; r < RB; ++r) a[i][e][r] = make_uint4(0, 0, 0, 0);
#pragma unroll
          for (int n = 0; n < NB; ++n) b[e][n] = make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < RB; ++r) {
#pragma unroll
          for (int n = 0; n < NB; ++n) Chunk<BF16>::mma(acc[r * NACC + (n < NACC ? n : NACC - 1)], a[i][e][r], b[e][n]);
        }
      }
    }
  };
  int s0 = w * U;
  for (; (s0 + U) * 8 <= chunks; s0 += W * U) steps(s0, std::true_type{});
  if (s0 * 8 < chunks) steps(s0, std::false_type{});
}
template <bool BF16, int RB, int NB, int NACC, int W>
__device__ __forceinline__ void wave_tile(const uint4* const (&row)[RB], const uint4* const (&tok)[NB], int chunks, int w,
                                          f32x4 (&acc)[RB * NACC]) {
#pragma unroll
  for (int n = 0; n < RB * NACC; ++n) acc[n] = {0.f, 0.f, 0.f, 0.f};
  if (chunks >= 32 * W) wave_steps<BF16, RB, NB, NACC, W, 4>(row, tok, chunks, w, acc);
  else if (chunks >= 16 * W) wave_steps<BF16, RB, NB, NACC, W, 2>(row, tok, chunks, w, acc);
  else wave_steps<BF16, RB, NB, NACC, W, 1>(row, tok, chunks, w, acc);
}

// Sum of the W waves' tiles in wave order, on wave 0.
template <int W, int N>
__device__ __forceinline__ void add_tiles(f32x4 (&acc)[N], f32x4 (&lds)[W][N][64], int w, int l) {
#pragma unroll
  for (int n = 0; n < N; ++n) lds[w][n][l] = acc[n];
  __syncthreads();
  if (w == 0)
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int i = 1; i < W; ++i) acc[n] += lds[i][n][l];
}

}  // namespace omnimoe
