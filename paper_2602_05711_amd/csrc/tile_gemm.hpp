// Matrix products of the shared branch's training and adapter kernels: a workgroup's TM x TN tile of C = A B^T, the
// operands copied global -> LDS without registers, two stages, products on the matrix cores with fp32 accumulation
// (v_mfma_f32_32x32x16_bf16, or v_mfma_f32_32x32x2_f32 for fp32 layers).
//
// An operand is indexed (r, k): r a row of the product's result (its columns for B), k the summed index. It lies in
// memory either with k contiguous (element (r, k) at p[r ld + k]) or, MNC, with r contiguous (p[k ld + r]), so that
// the way back needs no transposed copies: the weights of the forward products are read as they are. A stage holds
// kStep(T) values of k (64 bf16, 32 fp32): 128 bytes a row either way.
//   k contiguous: rows of 128 bytes; the 16-byte chunk j of row r lies at j ^ ((r >> 1) & 7), so that the rows read by
//     one operand load fall in distinct banks.
//   MNC bf16: rows k of 2 R bytes; a lane's eight k values come from two ds_read_b64_tr_b16, each of which hands the
//     lanes of a 16-lane group one column each of a 4 (k) x 16 (r) block; the 64-byte chunks of row k are permuted by
//     its low bits, so that a block's four rows fall in distinct banks.
//   MNC fp32: rows k of 4 R bytes, read value by value; the 128-byte chunks alternate with bit 2 of k.
// The sum's last stage may be partial: chunks past K are copied from a chunk of zeros. Rows past the operand's last one
// read that row again (their results are not stored).
//
// A 256 x 256 tile of eight waves moves 256 KiB through the LDS port in a stage (64 in, 192 out), 2048 cycles, as long as
// its products take on the matrix cores: 1.14 PFLOP/s in the weight gradients' long sums (d = d_ff = 2048, 16384 tokens),
// 0.87 in dx and the adapters' gate and up projection (sums of 4096 and 2048, one or two rounds of tiles whose ends nothing
// covers), where the library's products of these sizes reach 1.2 to 1.4. Four waves of 128 x 128, four stages of half the depth, copies spread over the stage and an epilogue through LDS
// were no faster. Small tiles run at the rate at which L2 fills LDS (9.5 to 11.6 TB/s).
#pragma once

#include "device_common.hpp"
#include "internal.hpp"

namespace omnimoe {

typedef __bf16 tg_bf16x8 __attribute__((ext_vector_type(8)));
typedef float tg_f32x4 __attribute__((ext_vector_type(4)));
typedef float tg_f32x16 __attribute__((ext_vector_type(16)));
typedef short tg_s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void* tg_lds_ptr;
typedef __attribute__((address_space(3))) tg_s16x4* tg_lds_s16x4;

static __device__ const uint4 tile_zeros = {0, 0, 0, 0};  // what is copied in place of chunks past K

struct BF16 {
  typedef uint16_t elem;
  typedef tg_bf16x8 frag;
  static constexpr int kSize = 2, kStep = 64, kMma = 1;
};
struct F32 {
  typedef float elem;
  typedef tg_f32x4 frag;
  static constexpr int kSize = 4, kStep = 32, kMma = 4;
};

// acc += (rows of a) x (rows of b): register q of lane l is a's row 8 (q / 4) + 4 (l / 32) + q % 4 and b's row
// l % 32.
__device__ __forceinline__ void tile_mma(tg_f32x16& acc, tg_bf16x8 a, tg_bf16x8 b) {
  acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0);
}
__device__ __forceinline__ void tile_mma(tg_f32x16& acc, tg_f32x4 a, tg_f32x4 b) {
#pragma unroll
  for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], acc, 0, 0, 0);
}

constexpr int64_t kTileReach = int64_t(1) << 32;  // bytes that a tile's 32-bit offsets count
static_assert(256LL * 2 * kMaxFeatures * 4 < kTileReach, "256 rows");
static_assert(2LL * kMaxFeatures * kMaxWidth * 2 < kTileReach && 2LL * kMaxFeatures * kMaxWidthF32 * 4 < kTileReach, "w_gu");

// One operand's R rows of a stage, copied by NW waves.
template <class T, int R, bool MNC, int NW>
struct TileOperand {
  static constexpr int kBytes = R * 128;
  static constexpr int kCopies = R / 8 / NW;  // 1 KiB each
  static_assert(R % (8 * NW) == 0, "each wave copies whole KiB");
  static constexpr int kReads = !MNC ? 1 : T::kSize;         // LDS reads of a fragment (MNC bf16: 2, fp32: 4)
  static constexpr int kPer = 16 / T::kSize;                 // elements per 16-byte chunk
  static constexpr int kRowChunks = MNC ? R / kPer : 8;      // 16-byte chunks per LDS row
  typedef typename T::elem elem;

  // Copy i of stage kt reads from base + kt step + off[i] (bytes; base and step are the same on every lane). off is less
  // than 4 GiB: it reaches over 256 rows, or 64 of the summed index, of at most 2 kMaxFeatures values, over all of w_gu (up
  // rows beside gate rows) or w_down, or over the rows of x of an adapters' pass (a static_assert each).
  const char* base;
  int64_t step;
  uint32_t off[kCopies];
  int lds;  // this wave's first byte within the operand

  // Position of chunk c in LDS row `row` (an involution in c).
  static __device__ __forceinline__ int place(int row, int c) {
    if constexpr (!MNC) return c ^ ((row >> 1) & 7);
    else if constexpr (T::kSize == 4) return c ^ (((row >> 2) & 1) << 3);
    else if constexpr (R >= 128) return c ^ ((row & 3) << 2);
    else return c ^ (((row >> 1) & 1) << 2);
  }

  // row(r): the operand's row in memory of tile row r (0 <= r < R); for MNC it must keep groups of kPer together.
  template <class Row>
  __device__ __forceinline__ void init(const elem* p, int64_t ld, int wid, int lane, Row row) {
    base = (const char*)p;
    step = (MNC ? (int64_t)T::kStep * ld : T::kStep) * T::kSize;
    lds = wid * kCopies * 1024;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int at = (wid * kCopies + i) * 64 + lane;  // 16-byte position within the operand
      const int lrow = at / kRowChunks, c = place(lrow, at % kRowChunks);
      const int64_t e = MNC ? (int64_t)lrow * ld + row(c * kPer) : (int64_t)row(lrow) * ld + c * kPer;
      off[i] = (uint32_t)(e * T::kSize);
    }
  }
  // k of this lane's chunk in copy i, within the stage
  static __device__ __forceinline__ int chunk_k(int i, int lane, int wid) {
    const int at = (wid * kCopies + i) * 64 + lane;
    const int lrow = at / kRowChunks;
    return MNC ? lrow : place(lrow, at % kRowChunks) * kPer;
  }
  // Stage kt of a sum over K values of k that starts `skip` bytes past base.
  __device__ __forceinline__ void copy(unsigned char* st, int at, int64_t skip, int kt, int K, int wid, int lane) const {
    const int to = at + lds;
    const char* const from = base + skip + kt * step;
    if ((kt + 1) * T::kStep <= K) {
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        uint32_t o = off[i];
        asm volatile("" : "+v"(o));  // (kept 32 bits wide: the address is a scalar base and an offset)
        __builtin_amdgcn_global_load_lds((const void*)(from + o), (tg_lds_ptr)(st + (to + i * 1024)), 16, 0, 0);
      }
    } else {
      int l = lane;
      asm volatile("" : "+v"(l));  // nothing of this branch is worth a register in the loop
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        uint32_t o = off[i];
        asm volatile("" : "+v"(o));
        const char* const p = kt * T::kStep + chunk_k(i, l, wid) < K ? from + o : (const char*)&tile_zeros;
        __builtin_amdgcn_global_load_lds((const void*)p, (tg_lds_ptr)(st + (to + i * 1024)), 16, 0, 0);
      }
    }
  }
  // Rows r0 .. r0 + 31 (r0 a multiple of 32), quarter ks of the stage; the operand starts `at` bytes into the array st.
  // (One offset from the array: through a longer chain of them the compiler loses sight of which array is read.)
  static __device__ __forceinline__ typename T::frag frag(const unsigned char* st, int at, int r0, int ks, int lane) {
    if constexpr (!MNC) {
      const int r = r0 + (lane & 31);
      return *(const typename T::frag*)(st + (at + r * 128 + (((ks * 2 + (lane >> 5)) ^ ((r >> 1) & 7)) << 4)));
    } else if constexpr (T::kSize == 2) {
      const int g = lane >> 4, i = lane & 15;
      const int k = ks * 16 + (g >> 1) * 8 + (i >> 2);
      const int o = at + k * (2 * R) + place(k, r0 / 8 + (g & 1) * 2 + ((i & 3) >> 1)) * 16 + (i & 1) * 8;
      const tg_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tg_lds_s16x4)(st + o));
      const tg_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((tg_lds_s16x4)(st + (o + 4 * (2 * R))));
      typedef short s16x8 __attribute__((ext_vector_type(8)));
      const s16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
      return __builtin_bit_cast(tg_bf16x8, v);
    } else {
      const int k = ks * 8 + (lane >> 5) * 4, r = r0 + (lane & 31);
      const int o = at + k * (4 * R) + place(k, r / 4) * 16 + (r & 3) * 4;
      tg_f32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = *(const float*)(st + (o + e * (4 * R)));
      return v;
    }
  }
};

// One or two ranges of the summed index: K values each, a_skip and b_skip bytes past the operands' bases.
struct TileRange {
  int K;
  int64_t a_skip, b_skip;
};

// The workgroup's sum over the ranges into acc[i][j]: a's rows a0[i] .. + 31 and b's rows b0[j] .. + 31 of the tile.
// st0 and st1 hold a stage of both operands each. They are two __shared__ arrays and every access names one of them
// (the loop is unrolled by two for it): the compiler knows which array a copy in flight writes only by its name, and
// makes a read that might touch it wait for all copies. Every thread of the workgroup takes part; on return the LDS is
// free.
//
// Stage s + 2 is requested as soon as the last quarter of stage s is in every wave's registers, and the first quarter of
// stage s + 1 is read before that last quarter's products: behind the one barrier of a stage the matrix cores still have
// a quarter to work on, and a stage's copies have a whole stage's products to arrive in.
template <class T, class OA, class OB, int MI, int NJ>
__device__ __forceinline__ void tile_sum(const OA& a, const OB& b, const TileRange (&range)[2], const int (&a0)[MI],
                                         const int (&b0)[NJ], unsigned char* st0, unsigned char* st1, int wid, int lane,
                                         tg_f32x16 (&acc)[MI][NJ]) {
  const int n0 = (range[0].K + T::kStep - 1) / T::kStep, n1 = (range[1].K + T::kStep - 1) / T::kStep;
  const int n = (n0 + n1 + 1) & ~1;  // an odd number of stages ends with one of zeros
  if (n == 0) return;
  auto copy = [&](unsigned char* st, int s) {
    const TileRange& r = s < n0 ? range[0] : range[1];
    const int kt = s < n0 ? s : s - n0;
    a.copy(st, 0, r.a_skip, kt, r.K, wid, lane);
    b.copy(st, OA::kBytes, r.b_skip, kt, r.K, wid, lane);
  };
  // (a barrier alone does not wait for copies that go past the registers)
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
  // products of one quarter with the next one's reads between them
  constexpr int kReads = MI * OA::kReads + NJ * OB::kReads, kMma = MI * NJ * T::kMma;
  constexpr int kPer = (kReads + kMma - 1) / kMma;
  auto interleave = [&]() {
#pragma unroll
    for (int i = 0; i < kMma; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x100, kPer, 0);  // LDS reads
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);     // a product
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto stage = [&](unsigned char* cur, unsigned char* next, int s) {
    __builtin_amdgcn_sched_barrier(0);
    read(cur, 1);
    mma(0);
    interleave();
    read(cur, 2);
    mma(1);
    interleave();
    read(cur, 3);
    mma(2);
    interleave();
    // the wave's copies of stage s + 1 and its reads of stage s are done, and with the barrier everyone's
    wait_copies();
    __syncthreads();
    if (s + 2 < n) copy(cur, s + 2);
    __builtin_amdgcn_sched_barrier(0);
    read(next, 0);  // (after the last stage: what is there, unused)
    mma(3);
    interleave();
  };
  copy(st0, 0);
  wait_copies();
  __syncthreads();
  copy(st1, 1);
  read(st0, 0);
#pragma unroll 1
  for (int s = 0; s < n; s += 2) {
    stage(st0, st1, s);
    stage(st1, st0, s + 1);
  }
  __syncthreads();
}

template <int MI, int NJ>
__device__ __forceinline__ void tile_zero(tg_f32x16 (&acc)[MI][NJ]) {
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;
}

// Four neighbouring values in the layer's type.
__device__ __forceinline__ void store4(uint16_t* p, float a, float b, float c, float d) {
  uint2 o;
  o.x = (uint32_t)bf16_rne(a) | ((uint32_t)bf16_rne(b) << 16);
  o.y = (uint32_t)bf16_rne(c) | ((uint32_t)bf16_rne(d) << 16);
  *(uint2*)p = o;
}
__device__ __forceinline__ void store4(float* p, float a, float b, float c, float d) {
  *(float4*)p = make_float4(a, b, c, d);
}

}  // namespace omnimoe
