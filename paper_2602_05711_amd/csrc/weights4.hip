// Weights in 4 bits and their products with a few rows an expert.
//
// A block of 32 values of a row is e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6, and a sign) times a power of two 2^s, s the
// least with max |w| <= 6 2^s: v_cvt_scalef32_pk_bf16_fp4 turns two codes and the scale into two bf16 values, exactly, so
// that no product needs a scale of its own and the sums run through all of a row.
#include "few_tile.hpp"
#include "grouped_rows.hpp"
#include "internal.hpp"
#include "tile_gemm.hpp"
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

// A block a thread: bound by memory, laid out once.
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
  const int32_t *offsets, *perm;
  int N, M, k, n, hk, x_order, y_order;
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

// 16 RB weight rows (SWIGLU: half of them gate rows, in turn) for a unit of up to sixteen positions. A step is 128 values
// of k, a block of 32 a lane (16 bytes of codes and their scale); a workgroup's waves take steps in turn, U at a time in
// flight, and their tiles are added in wave order.
template <bool BF16, int RB, bool SWIGLU, int U>
__global__ __launch_bounds__(256) void product4_kernel(Product4Args p, int groups) {
  constexpr int W = 4, kSize = BF16 ? 2 : 4, FB = SWIGLU ? RB / 2 : RB, kChunks = Codes8<BF16>::kChunks;
  typedef typename std::conditional<BF16, uint16_t, float>::type elem;
  __shared__ f32x4 tiles[W][RB][64];
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quad = l >> 4;
  const int want = blockIdx.x / (unsigned)groups, f0 = (int)(blockIdx.x % (unsigned)groups) * 16 * FB;
  RowUnit u;
  if (find_unit<256>(p.offsets, p.N, p.M, 16, (int*)tiles, [&](int) { return want; }, u) <= want) return;
  __syncthreads();
  const int at = row_of(p.perm, p.x_order, p.hk, p.M, u.first + ((l & 15) < u.count ? (l & 15) : u.count - 1));
  const char* const tok = (const char*)p.x + (int64_t)(at < 0 ? 0 : at) * p.k * kSize;
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
  for (int s0 = w * U; s0 * 4 < nb; s0 += W * U) {
    uint4 code[U][RB];
    float scale[U][RB];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int block = (s0 + i) * 4 + quad, there = block < nb ? block : nb - 1;
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        code[i][b] = *(const uint4*)(p.codes + (row[b] + there) * 16);
        scale[i][b] = __uint_as_float((uint32_t)p.scales[row[b] + there] << 23);
        if (block >= nb) {
          code[i][b] = make_uint4(0, 0, 0, 0);
          scale[i][b] = 1.0f;
        }
      }
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int block = (s0 + i) * 4 + quad, there = block < nb ? block : nb - 1;
      uint4 x[kChunks];
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        x[c] = *(const uint4*)(tok + (int64_t)there * 32 * kSize + c * 16);
        if (block >= nb) x[c] = make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        Codes8<BF16>::mma(acc[b], code[i][b].x, scale[i][b], x, 0);
        Codes8<BF16>::mma(acc[b], code[i][b].y, scale[i][b], x, 1);
        Codes8<BF16>::mma(acc[b], code[i][b].z, scale[i][b], x, 2);
        Codes8<BF16>::mma(acc[b], code[i][b].w, scale[i][b], x, 3);
      }
    }
  }
  add_tiles(acc, tiles, w, l);
  if (w || (l & 15) >= u.count) return;
  const int to = row_of(p.perm, p.y_order, p.hk, p.M, u.first + (l & 15));
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
      if constexpr (SWIGLU) v[e] = activation(1, v[e]) * acc[b + 1][e];
    }
    store4(out + f, v[0], v[1], v[2], v[3]);
  }
}

template <bool BF16, bool SWIGLU>
hipError_t product4(const Product4Args& p, hipStream_t st) {
  constexpr int RB = 2, U = 2;
  const int64_t units = p.M / 16 + p.N < p.M ? p.M / 16 + p.N : p.M, per = SWIGLU ? 8 * RB : 16 * RB;
  const int64_t groups = (p.n + per - 1) / per, grid = units * groups;
  if (grid > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((product4_kernel<BF16, RB, SWIGLU, U>), dim3((unsigned)grid), dim3(256), 0, st, p, (int)groups);
  return hipGetLastError();
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
  const Product4Args p{x, codes, scales, y, offsets, perm, (int)s.N, (int)s.M, q.n_in, q.n_out, s.hk, q.x_order, q.y_order};
  if (s.bf16) return q.swiglu ? product4<true, true>(p, st) : product4<true, false>(p, st);
  return q.swiglu ? product4<false, true>(p, st) : product4<false, false>(p, st);
}

}  // namespace omnimoe
