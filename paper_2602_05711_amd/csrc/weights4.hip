// Weights in 4 bits and their products with a few rows an expert.
//
// A block of 32 values of a row is e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6, and a sign) times a power of two 2^s, s the
// least with max |w| <= 6 2^s: v_cvt_scalef32_pk_bf16_fp4 turns two codes and the scale into two bf16 values, exactly, so
// that no product needs a scale of its own and the sums run through all of a row.
//
// The products are bound by reading the codes once: 128 rows on 64 experts of 2048 x 2048 with SwiGLU 28 to 32 us, 4.2 TB/s (a
// kernel that only reads as many codes and scales in this order 21 us); eight rows of one token 7.4 us. What cost most was a byte
// load for each scale (42 us); a row's scales of several steps come in one where the rows are of whole steps. Other widths have the
// byte loads: 64 experts of 2048 x 2304 45 us, 2880 45, 768 22 (1024: 21).
#include "few_tile.hpp"
#include "grouped_rows.hpp"
#include "internal.hpp"
#include "vec8.hpp"

namespace omnimoe {
namespace {

typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// Least s with -125 <= s <= 125 and amax <= 6 2^s: amax = m 2^k with 1 <= m < 2 and 6 = 1.5 2^2, so s = k - 2, one more
// where m > 1.5.
__device__ __forceinline__ int block_exponent4(uint32_t amax_bits) {
  const int k = (int)(amax_bits >> 23) - 127, s = k - 2 + ((amax_bits & 0x007FFFFFu) > 0x00400000u ? 1 : 0);
  return s < -125 ? -125 : s > 125 ? 125 : s;
}

// A block a thread: bound by memory, laid out once. 64 matrices of 2048 x 2048, bf16: 142 us, 4.8 TB/s, and load4_kernel 149, 4.6;
// of 1024 x 1024, fp32: 49 (from the caches in part) and 73.
template <bool BF16>
__global__ __launch_bounds__(256) void store4_kernel(const void* __restrict__ w, uint8_t* __restrict__ codes,
                                                     uint8_t* __restrict__ scales, int64_t blocks) {
  for (int64_t b = (int64_t)blockIdx.x * 256 + threadIdx.x; b < blocks; b += (int64_t)gridDim.x * 256) {
    float v[4][8];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      load8<BF16>(w, b * 32 + i * 8, v[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t a = __float_as_uint(v[i][e]) & 0x7FFFFFFFu;
        m = a > m ? a : m;
      }
    }
    const bool fine = m < 0x7F800000u;
    const int s = block_exponent4(m);
    uint32_t word[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      word[i] = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float a = ldexpf(fabsf(v[i][e]), -s);  // (exact where it is not far below the least border)
        const uint32_t c = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.0f);
        word[i] |= (c | (__float_as_uint(v[i][e]) >> 31 << 3)) << (4 * e);
      }
      if (!fine) word[i] = 0;
    }
    *(uint4*)(codes + b * 16) = make_uint4(word[0], word[1], word[2], word[3]);
    scales[b] = fine ? (uint8_t)(s + 127) : 255;
  }
}

__device__ __forceinline__ float code_value(uint32_t c) {
  const uint32_t m = c & 7u;
  const float v = m < 2 ? 0.5f * (float)m : ldexpf(1.0f + 0.5f * (float)(m & 1u), (int)(m >> 1) - 1);
  return c & 8u ? -v : v;
}

template <bool BF16>
__global__ __launch_bounds__(256) void load4_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                    void* __restrict__ w, int64_t blocks) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < blocks * 4; i += (int64_t)gridDim.x * 256) {
    const uint32_t word = *(const uint32_t*)(codes + i * 4);
    const int byte = scales[i >> 2];
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      v[e] = byte == 255 ? __uint_as_float(0x7FC00000u) : ldexpf(code_value(word >> (4 * e) & 15u), byte - 127);
    store8<BF16>(w, i * 8, v);
  }
}

struct Product4Args {
  const void* x;
  const uint8_t *codes, *scales;
  void* y;
  const int32_t* offsets;
  int N, M, k, n;
  RowOrder x_rows, y_rows;
  unsigned block0;
};

// Eight codes of a lane's block against eight values of each operand's block.
template <bool BF16>
struct Codes8;
template <>
struct Codes8<true> {
  static constexpr int kChunks = 4;  // 16-byte chunks of a block of x
  static __device__ __forceinline__ void mma(f32x4& acc, uint32_t word, float scale, const uint4* x, int i) {
    union {
      bf16x2v pair[4];
      bf16x8 all;
    } a;
    a.pair[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 0);
    a.pair[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 1);
    a.pair[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 2);
    a.pair[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, 3);
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.all, __builtin_bit_cast(bf16x8, x[i]), acc, 0, 0, 0);
  }
};
template <>
struct Codes8<false> {
  static constexpr int kChunks = 8;
  static __device__ __forceinline__ void mma(f32x4& acc, uint32_t word, float scale, const uint4* x, int i) {
    const f32x2 a[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, 0),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, 2),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, 3)};
    const uint4 lo = x[2 * i], hi = x[2 * i + 1];
    const uint32_t b[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int e = 0; e < 8; ++e)
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e >> 1][e & 1], __uint_as_float(b[e]), acc, 0, 0, 0);
  }
};

// The scale bytes of U steps of a lane's row (4 U neighbouring blocks, WIDE: one aligned load, the same on the row's four
// lanes), and a step's as the float 2^s of this lane's block.
template <int U, bool WIDE>
struct Scales {
  uint32_t word[U];
  __device__ __forceinline__ void load(const uint8_t* row, int block, int quad, int last) {
    if constexpr (WIDE) {
      if constexpr (U == 4) {
        const uint4 v = *(const uint4*)(row + block);
        word[0] = v.x, word[1] = v.y, word[2] = v.z, word[3] = v.w;
      } else if constexpr (U == 2) {
        const uint2 v = *(const uint2*)(row + block);
        word[0] = v.x, word[1] = v.y;
      } else {
        word[0] = *(const uint32_t*)(row + block);
      }
    } else {
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int at = block + 4 * i + quad;
        word[i] = row[at < last ? at : last];
      }
    }
  }
  __device__ __forceinline__ float of(int i, int quad) const {
    const uint32_t v = WIDE ? word[i] >> (8 * quad) : word[i];
    return __uint_as_float((v << 23) & 0x7F800000u);
  }
};

// 16 RB weight rows (SWIGLU: half of them gate rows, in turn) for a unit of up to sixteen positions. A step is 128 values
// of k, a block of 32 a lane (16 bytes of codes); a workgroup's W waves take U neighbouring steps in turn, all of their codes
// and scales in flight together, and their tiles are added in wave order.
template <bool BF16, int RB, bool SWIGLU, int W, int U, bool WIDE>
__global__ __launch_bounds__(64 * W) void product4_kernel(Product4Args p, int groups) {
  constexpr int kSize = BF16 ? 2 : 4, FB = SWIGLU ? RB / 2 : RB, kChunks = Codes8<BF16>::kChunks;
  typedef typename std::conditional<BF16, uint16_t, float>::type elem;
  __shared__ f32x4 tiles[W][RB][64];
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quad = l >> 4;
  const unsigned block = p.block0 + blockIdx.x;
  const int want = block / (unsigned)groups, f0 = (int)(block % (unsigned)groups) * 16 * FB;
  RowUnit u;
  if (find_unit<64 * W>(p.offsets, p.N, p.M, 16, (int*)tiles, [&](int) { return want; }, u) <= want) return;
  __syncthreads();
  const int pos = u.first + ((l & 15) < u.count ? (l & 15) : u.count - 1), task = p.x_rows.task(pos);
  const int nb = p.k / 32;
  int64_t row[RB];  // blocks before this lane's weight rows
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const int f = f0 + 16 * (SWIGLU ? b / 2 : b) + (l & 15), c = f < p.n ? f : p.n - 1;
    row[b] = ((int64_t)u.expert * (SWIGLU ? 2 : 1) * p.n + (SWIGLU && (b & 1) ? p.n + c : c)) * nb;
  }
  f32x4 acc[RB];
#pragma unroll
  for (int b = 0; b < RB; ++b) acc[b] = {0.f, 0.f, 0.f, 0.f};
  auto steps = [&](int s0, auto whole) {
    constexpr bool kWhole = decltype(whole)::value;
    uint4 code[U][RB];
    Scales<U, WIDE> scale[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      scale[b].load(p.scales + row[b], s0 * 4, quad, nb - 1);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int block = (s0 + i) * 4 + quad;
        code[i][b] = *(const uint4*)(p.codes + (row[b] + (kWhole || block < nb ? block : nb - 1)) * 16);
      }
    }
    const int at = p.x_rows.of(pos, task);
    const char* const tok = (const char*)p.x + (int64_t)(at < 0 ? 0 : at) * p.k * kSize;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int block = (s0 + i) * 4 + quad;
      const bool there = kWhole || block < nb;
      uint4 x[kChunks];
#pragma unroll
      for (int c = 0; c < kChunks; ++c) x[c] = *(const uint4*)(tok + (int64_t)(there ? block : nb - 1) * 32 * kSize + c * 16);
      if (!there)  // (both operands: an infinity times a zero would not be one)
#pragma unroll
        for (int c = 0; c < kChunks; ++c) x[c] = make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        const float f = there ? scale[b].of(i, quad) : 1.0f;
        const uint4 q = there ? code[i][b] : make_uint4(0, 0, 0, 0);
        Codes8<BF16>::mma(acc[b], q.x, f, x, 0);
        Codes8<BF16>::mma(acc[b], q.y, f, x, 1);
        Codes8<BF16>::mma(acc[b], q.z, f, x, 2);
        Codes8<BF16>::mma(acc[b], q.w, f, x, 3);
      }
    }
  };
  int s0 = w * U;
  for (; (s0 + U) * 4 <= nb; s0 += W * U) steps(s0, std::true_type{});
  if (s0 * 4 < nb) steps(s0, std::false_type{});
  add_tiles(acc, tiles, w, l);
  if (w || (l & 15) >= u.count) return;
  const int to = p.y_rows.of(pos, task);
  if (to < 0) return;
  elem* const out = (elem*)p.y + (int64_t)to * p.n;
#pragma unroll
  for (int b = 0; b < RB; b += SWIGLU ? 2 : 1) {
    const int f = f0 + 16 * (SWIGLU ? b / 2 : b) + 4 * quad;
    if (f >= p.n) break;
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = acc[b][e];
      if constexpr (SWIGLU) v[e] = swiglu<BF16>(v[e], acc[b + (SWIGLU ? 1 : 0)][e]);
    }
    put4(out + f, v[0], v[1], v[2], v[3]);
  }
}

template <bool BF16, bool SWIGLU, int RB, int W, int U>
hipError_t product4_launch(const Product4Args& p, int64_t units, hipStream_t st) {
  const int64_t per = SWIGLU ? 8 * RB : 16 * RB, groups = (p.n + per - 1) / per, grid = units * groups;
  if (p.k / 32 % (4 * U) == 0)
    return launch_numbered(product4_kernel<BF16, RB, SWIGLU, W, U, true>, grid, 64 * W, st, p, (int)groups);
  return launch_numbered(product4_kernel<BF16, RB, SWIGLU, W, U, false>, grid, 64 * W, st, p, (int)groups);
}

// Row blocks a workgroup: four where that leaves a thousand workgroups (four a compute unit), two from 256 on, or one (the
// SwiGLU's two), with the steps spread over eight waves. 64 experts, n_in = 2048, n_out = 1024, SwiGLU: 16 tokens 29.6 us
// with four blocks and 32.3 with two, one token 8.6 and 7.7; one matrix of 2048 x 8192, one token: 18.3, 12.0 and, with
// one, 7.8 us. fp32 weights keep the matrix cores busy (eight products for one of bf16): one block, 7 tokens,
// 2080 x 2056: 7.5 us, with two blocks on four waves 10.5.
template <bool BF16, bool SWIGLU>
hipError_t product4(const Product4Args& p, hipStream_t st) {
  const int64_t units = p.M / 16 + p.N < p.M ? p.M / 16 + p.N : p.M, blocks = units * (((SWIGLU ? 2 : 1) * p.n + 15) / 16);
  constexpr int kLeast = SWIGLU ? 2 : 1;
  if constexpr (BF16) {
    if (blocks >= 4096) return product4_launch<true, SWIGLU, 4, 4, 4>(p, units, st);
    if (blocks >= 512) return product4_launch<true, SWIGLU, 2, 4, 2>(p, units, st);
    return product4_launch<true, SWIGLU, kLeast, 8, 2>(p, units, st);
  } else {
    return product4_launch<false, SWIGLU, kLeast, 8, 1>(p, units, st);
  }
}

unsigned grid_of(int64_t threads) {
  const int64_t b = (threads + 255) / 256;
  return (unsigned)(b > 65536 ? 65536 : b);
}

int64_t all_blocks(const Shape& s, const ProductShape& q) { return s.N * (q.swiglu ? 2 : 1) * q.n_out * (q.n_in / 32); }

}  // namespace

hipError_t launch_weights4_store(const Shape& s, const ProductShape& q, const void* w, uint8_t* codes, uint8_t* scales,
                                 hipStream_t st) {
  const int64_t n = all_blocks(s, q);
  if (s.bf16) hipLaunchKernelGGL(store4_kernel<true>, dim3(grid_of(n)), dim3(256), 0, st, w, codes, scales, n);
  else hipLaunchKernelGGL(store4_kernel<false>, dim3(grid_of(n)), dim3(256), 0, st, w, codes, scales, n);
  return hipGetLastError();
}

hipError_t launch_weights4_load(const Shape& s, const ProductShape& q, const uint8_t* codes, const uint8_t* scales, void* w,
                                hipStream_t st) {
  const int64_t n = all_blocks(s, q);
  if (s.bf16) hipLaunchKernelGGL(load4_kernel<true>, dim3(grid_of(n * 4)), dim3(256), 0, st, codes, scales, w, n);
  else hipLaunchKernelGGL(load4_kernel<false>, dim3(grid_of(n * 4)), dim3(256), 0, st, codes, scales, w, n);
  return hipGetLastError();
}

hipError_t launch_grouped_product4(const Shape& s, const ProductShape& q, const void* x, const uint8_t* codes,
                                   const uint8_t* scales, const int32_t* offsets, const int32_t* perm, void* y,
                                   hipStream_t st) {
  const Product4Args p{x, codes, scales, y, offsets, (int)s.N, (int)s.M, q.n_in, q.n_out,
                       RowOrder::make(perm, (int)s.M, q.x_order, s.hk), RowOrder::make(perm, (int)s.M, q.y_order, s.hk), 0};
  if (s.bf16) return q.swiglu ? product4<true, true>(p, st) : product4<true, false>(p, st);
  return q.swiglu ? product4<false, true>(p, st) : product4<false, false>(p, st);
}

}  // namespace omnimoe
