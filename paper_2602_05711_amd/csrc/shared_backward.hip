// The way back through the shared branch MLP(x) = W_down (silu(W_g x) (.) (W_u x)) (Eq. 7's SwiGLU block) from the
// 8-bit checkpoint of its input x~:
//   g = W_g x~, u = W_u x~, p = 1 / (1 + exp(-g)), a = g p u, da = W_down^T dy
//   dg = da u p (1 + g (1 - p)), du = da g p
//   dx = dx_in + W_g^T dg + W_u^T du,  dW_g = dg x~^T, dW_u = du x~^T, dW_down = dy a^T (sums over the tokens)
// Four launches: the checkpoint's and dy's values in the layer's type; the three products that a tile of dg, du and a
// needs, whose sums meet in registers; dx and the weight gradients (large tiles: a launch each), split over the summed
// index (the tokens; for dx of few tokens the features) into fp32 partial sums that a last launch adds in order. No atomics: the result is the same on every run. Sums
// are fp32. bf16 layers round a, dg and du to bf16 (once each, to nearest) for the matrix cores, as the forward pass rounds
// a; dy, fp32 from the caller, enters as two bf16 values, its rounding and what that leaves (2^-17 relative), for two
// products more: with dy rounded as well, three roundings (dy, a or dg, the result) put the weight gradients 0.0029 of
// their norm from the exact ones instead of 0.0023, the rounding of the result alone being 0.0017. Where a weight of W_down
// or a value of a is infinite, the two values' products can meet as infinities of either sign or as zero times it: NaN
// instead of an infinity (keeping them apart would take da's accumulators twice).
#include "bf16_parts.hpp"
#include "checkpoint.hpp"
#include "internal.hpp"
#include "tile_gemm.hpp"

namespace omnimoe {
namespace {

// The bf16 operands: the checkpoint's values to x, and dy to hi = bf16(dy) and lo = bf16(dy - hi), eight of each a thread
// (bf16_part: hi is finite where dy is, lo zero where it is not). Bound by memory: [16384, 2048] 59 us, 6.3 TB/s. A pass
// of its own, because the tiles' operands are copied to LDS without passing registers.
__global__ __launch_bounds__(256) void operands_kernel(const uint8_t* __restrict__ codes,
                                                       const uint8_t* __restrict__ scales, const float* __restrict__ dy,
                                                       uint16_t* __restrict__ x, uint16_t* __restrict__ hi,
                                                       uint16_t* __restrict__ lo, int64_t T, int d) {
  const int q8 = d / 8, nblk = (d + 31) / 32;
  const int64_t n8 = T * q8;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n8; i += (int64_t)gridDim.x * 256) {
    const float4 a = *(const float4*)(dy + i * 8), b = *(const float4*)(dy + i * 8 + 4);
    const int64_t t = i / q8;
    const int c = (int)(i - t * q8);
    checkpoint_load8<true>(codes + i * 8, scales[t * nblk + (c >> 2)], x, i * 8);
    float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    uint32_t h[4], l[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      h[e] = bf16_part(v[2 * e]);
      h[e] |= bf16_part(v[2 * e + 1]) << 16;
      l[e] = (uint32_t)bf16_rne(v[2 * e]) | ((uint32_t)bf16_rne(v[2 * e + 1]) << 16);
    }
    *(uint4*)(hi + i * 8) = make_uint4(h[0], h[1], h[2], h[3]);
    *(uint4*)(lo + i * 8) = make_uint4(l[0], l[1], l[2], l[3]);
  }
}

struct HiddenArgs {
  const void *x, *dy, *dy_lo, *w_gu, *w_down;  // [T, d] three times (dy_lo: bf16 only), [2 F, d], [d, F]
  void *dh, *act;                      // [T, 2 F] (dg then du), [T, F]
  int64_t T;
  int d, F;
};

// TM tokens x FN features a workgroup; a wave holds 32 MJ tokens x 32 FI features of each of g, u and da (bf16: da in two
// passes, dy's two halves). Large tiles are bound by the LDS port (a stage's copies and reads take as long as its
// products): 16384 tokens, d = d_ff = 2048, 697 us, 0.79 PFLOP/s of the 4 x 137 GFLOP. Small ones run at L2's rate: 4093
// tokens, d = d_ff = 512, 24.9 us, 9.4 TB/s; fp32, 1000 tokens, 520, 40 us (64 us on 128 x 64).
template <class T, int TM, int FN, int WR, int WC>
__global__ __launch_bounds__(64 * WR * WC) void hidden_kernel(HiddenArgs p) {
  constexpr int NW = WR * WC, MJ = TM / WR / 32, FI = FN / WC / 32;
  typedef typename T::elem elem;
  __shared__ __attribute__((aligned(1024))) unsigned char st0[(2 * FN + TM) * 128], st1[(2 * FN + TM) * 128];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wid / WC, wc = wid % WC;
  const int F = p.F, tiles_f = (F + FN - 1) / FN;
  const int64_t m0 = (int64_t)(blockIdx.x / (unsigned)tiles_f) * TM;
  const int f0 = (int)(blockIdx.x % (unsigned)tiles_f) * FN;
  const int mlast = (int)((p.T - 1 < m0 + TM - 1 ? p.T - 1 : m0 + TM - 1) - m0);
  auto token = [&](int r) { return r < mlast ? r : mlast; };

  int b0[MJ], a2[2 * FI], a1[FI];
#pragma unroll
  for (int j = 0; j < MJ; ++j) b0[j] = (wr * MJ + j) * 32;
#pragma unroll
  for (int i = 0; i < FI; ++i) {
    a1[i] = a2[2 * i] = (wc * FI + i) * 32;
    a2[2 * i + 1] = FN + a1[i];
  }
  tg_f32x16 gu[2 * FI][MJ], da[FI][MJ];
  tile_zero(gu);
  tile_zero(da);
  TileOperand<T, TM, false, NW> x;  // rows of x~, then of dy: both [T, d]
  x.init((const elem*)p.x + m0 * p.d, p.d, wid, lane, token);
  {
    TileOperand<T, 2 * FN, false, NW> w;
    w.init((const elem*)p.w_gu, p.d, wid, lane, [&](int r) {
      const int f = f0 + (r < FN ? r : r - FN);
      return (f < F ? f : F - 1) + (r < FN ? 0 : F);
    });
    const TileRange all[2] = {{p.d, 0, 0}, {0, 0, 0}};
    tile_sum<T>(w, x, all, a2, b0, st0, st1, wid, lane, gu);
  }
  {
    TileOperand<T, FN, true, NW> w;
    w.init((const elem*)p.w_down, F, wid, lane, [&](int r) { return f0 + r < F ? f0 + r : F - w.kPer; });
    x.base = (const char*)((const elem*)p.dy + m0 * p.d);
    const TileRange both[2] = {{p.d, 0, 0}, {T::kSize == 2 ? p.d : 0, 0, (const char*)p.dy_lo - (const char*)p.dy}};
    tile_sum<T>(w, x, both, a1, b0, st0, st1, wid, lane, da);
  }
#pragma unroll
  for (int j = 0; j < MJ; ++j) {
    const int64_t t = m0 + b0[j] + (lane & 31);
    if (t >= p.T) continue;
    elem* const dh = (elem*)p.dh + t * 2 * F;
    elem* const act = (elem*)p.act + t * F;
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int f = f0 + a1[i] + 8 * q + 4 * (lane >> 5);
        if (f >= F) continue;
        float dg[4], du[4], a[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float g = gu[2 * i][j][4 * q + e], u = gu[2 * i + 1][j][4 * q + e], z = da[i][j][4 * q + e];
          const float s = 1.0f / (1.0f + expf(-g));
          a[e] = g * s * u;
          du[e] = z * (g * s);
          dg[e] = z * u * (s * (1.0f + g * (1.0f - s)));
        }
        store4(dh + f, dg[0], dg[1], dg[2], dg[3]);
        store4(dh + F + f, du[0], du[1], du[2], du[3]);
        store4(act + f, a[0], a[1], a[2], a[3]);
      }
  }
}

// C[m, n] = sum over k of B(m, k) A(n, k), a workgroup's tile TM x TN of one of up to three products and one part of
// its summed range. Parts (parts > 1) go to part[z][m, n] in fp32, whole sums to out in the layer's type, with add[m, n].
// With b_lo, B is b + b_lo: the range is run through twice, k in [K, 2 K) being b_lo's.
// Bound as hidden_kernel: 16384 tokens, d = d_ff = 2048, dx 321 us and the weight gradients 483 us, 0.86 and 1.14
// PFLOP/s.
struct Product {
  const void *a, *b, *b_lo;
  int64_t lda, ldb, M;
  int N, K, tiles_n, parts, kpart;
  int first;  // workgroup of the product's first tile
  void* out;
  const float* add;  // or NULL
  float* part;
};
struct ProductArgs {
  Product p[3];  // dx, dW_gu, dW_down
};
enum { kDx = 1, kWeights = 2 };  // the products of a launch

template <class T, int TM, int TN, int WR, int WC, bool B_MNC>
__device__ __forceinline__ void product_tile(const Product& p, int wg, unsigned char* st0, unsigned char* st1) {
  constexpr int NW = WR * WC, MJ = TM / WR / 32, NI = TN / WC / 32;
  typedef typename T::elem elem;
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wid / WC, wc = wid % WC;
  const int part = (wg - p.first) % p.parts, tile = (wg - p.first) / p.parts;
  const int n0 = tile % p.tiles_n * TN;
  const int64_t m0 = (int64_t)(tile / p.tiles_n) * TM;
  const int mlast = (int)((p.M - 1 < m0 + TM - 1 ? p.M - 1 : m0 + TM - 1) - m0);
  TileRange range[2];
  {
    const int64_t ka = p.lda * T::kSize, kb = (B_MNC ? p.ldb : 1) * T::kSize;
    const int64_t lo = (const char*)p.b_lo - (const char*)p.b;
    const int64_t k0 = (int64_t)part * p.kpart, k1 = p.parts == 1 ? 2 * (int64_t)p.K : k0 + p.kpart;
    auto cut = [&](int64_t v) { return (int)(v < 0 ? 0 : v > p.K ? p.K : v); };
    const int h0 = cut(k0), h1 = cut(k1), l0 = cut(k0 - p.K), l1 = p.b_lo ? cut(k1 - p.K) : l0;
    range[0] = {h1 - h0, h0 * ka, h0 * kb};
    range[1] = {l1 - l0, l0 * ka, l0 * kb + lo};
  }

  int a0[NI], b0[MJ];
#pragma unroll
  for (int j = 0; j < MJ; ++j) b0[j] = (wr * MJ + j) * 32;
#pragma unroll
  for (int i = 0; i < NI; ++i) a0[i] = (wc * NI + i) * 32;
  tg_f32x16 acc[NI][MJ];
  tile_zero(acc);
  TileOperand<T, TN, true, NW> a;
  TileOperand<T, TM, B_MNC, NW> b;
  a.init((const elem*)p.a, p.lda, wid, lane, [&](int r) { return n0 + r < p.N ? n0 + r : p.N - a.kPer; });
  if constexpr (B_MNC)
    b.init((const elem*)p.b + m0, p.ldb, wid, lane, [&](int r) { return r <= mlast ? r : mlast + 1 - b.kPer; });
  else
    b.init((const elem*)p.b + m0 * p.ldb, p.ldb, wid, lane, [&](int r) { return r < mlast ? r : mlast; });
  tile_sum<T>(a, b, range, a0, b0, st0, st1, wid, lane, acc);
#pragma unroll
  for (int j = 0; j < MJ; ++j) {
    const int64_t m = m0 + b0[j] + (lane & 31);
    if (m >= p.M) continue;
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int n = n0 + a0[i] + 8 * q + 4 * (lane >> 5);
        if (n >= p.N) continue;
        const int64_t at = m * p.N + n;
        float4 v = make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
        if (p.parts > 1) {
          *(float4*)(p.part + part * (p.M * p.N) + at) = v;
          continue;
        }
        if (p.add) {
          const float4 s = *(const float4*)(p.add + at);
          v.x += s.x;
          v.y += s.y;
          v.z += s.z;
          v.w += s.w;
        }
        store4((elem*)p.out + at, v.x, v.y, v.z, v.w);
      }
  }
}

// The workgroups of dx come before the weight gradients', each XCD having neighbouring tiles of both. Tiles below 256 x 256
// take them in one launch, since neither fills the compute units alone: 64 x 64 tiles, 4093 tokens, d = d_ff = 512, 32.8 us
// instead of 15.3 and 21.8 (on 128 x 128 tiles 25.1); fp32, 1000 tokens, 520, 44.5 instead of 27.8 and 24.8 (with dx in
// two parts 36.6).
template <class T, int TM, int TN, int WR, int WC, int WHICH>
__global__ __launch_bounds__(64 * WR * WC) void product_kernel(ProductArgs args) {
  __shared__ __attribute__((aligned(1024))) unsigned char st0[(TM + TN) * 128], st1[(TM + TN) * 128];
  const unsigned first = WHICH == kWeights ? 0 : WHICH == kDx ? gridDim.x : (unsigned)args.p[1].first;
  if (blockIdx.x < first) {
    if constexpr (WHICH & kDx)
      product_tile<T, TM, TN, WR, WC, false>(args.p[0], (int)xcd_contiguous(blockIdx.x, first), st0, st1);
  } else {
    if constexpr (WHICH & kWeights) {
      const int wg = (int)(first + xcd_contiguous(blockIdx.x - first, gridDim.x - first));
      product_tile<T, TM, TN, WR, WC, true>(args.p[wg >= args.p[2].first ? 2 : 1], wg, st0, st1);
    }
  }
}

// out = the parts' sum, in order (and add), of the products that have parts: n4[i] quads of p[i]. 4 to 9 us.
struct Quads {
  int64_t n4[3];
};
template <class T>
__global__ __launch_bounds__(256) void add_parts_kernel(ProductArgs args, Quads quads) {
  const int64_t all = quads.n4[0] + quads.n4[1] + quads.n4[2];
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int64_t first = quads.n4[0], second = first + quads.n4[1];
    const Product& p = args.p[i < first ? 0 : i < second ? 1 : 2];
    const int64_t at = (i - (i < first ? 0 : i < second ? first : second)) * 4, size = p.M * p.N;
    float4 v = *(const float4*)(p.part + at);
    auto sum = [&](const float* from) {
      const float4 s = *(const float4*)from;
      v.x += s.x;
      v.y += s.y;
      v.z += s.z;
      v.w += s.w;
    };
    for (int z = 1; z < p.parts; ++z) sum(p.part + z * size + at);
    if (p.add) sum(p.add + at);
    store4((typename T::elem*)p.out + at, v.x, v.y, v.z, v.w);
  }
}

size_t up(size_t v) { return (v + 255) & ~(size_t)255; }

int64_t tiles(int64_t M, int64_t N, int tm, int tn) { return ((M + tm - 1) / tm) * ((N + tn - 1) / tn); }

// How the weight gradients' sums over the tokens are split: parts of kpart values of k, dW_gu's range being the tokens
// and dW_down's twice those for bf16 (dy's two halves). Of the splits into 1 to 64 parts the one is taken that the
// workgroups' rounds over the compute units and the parts' way through memory make the shortest.
struct Parts {
  int gu, down, kpart;
};
Parts weight_parts(const Shape& s, int F, int tile) {
  if (s.T == 0) return {1, 1, 64};
  const int64_t tg = tiles(2 * (int64_t)F, s.d, tile, tile), td = tiles(s.d, F, tile, tile);
  const int64_t range = (s.bf16 ? 2 : 1) * s.T;
  // 256 compute units; smaller tiles' workgroups share one, two or four at a time
  const int64_t slots = tile == 256 ? 256 : tile == 128 ? 512 : 1024;
  // ns of a value of k in a tile, of a tile's start and end, of a KiB of a part written and read
  const double per_k = tile == 256 ? 55.0 : tile == 128 ? 16.0 : 12.0, fixed = 4000.0, per_kib = 0.5;
  Parts best{1, 1, 64};
  double least = 0;
  for (int n = 1; n <= 64; ++n) {
    const int64_t kpart = ((range + n - 1) / n + 63) / 64 * 64;
    const int pg = (int)((s.T + kpart - 1) / kpart), pd = (int)((range + kpart - 1) / kpart);
    const int64_t rounds = (tg * pg + td * pd + slots - 1) / slots;
    const double elems = (pg > 1 ? 2.0 * pg : 0.0) * F * s.d + (pd > 1 ? 1.0 * pd : 0.0) * F * s.d;
    const double ns = rounds * (kpart * per_k + fixed) + elems * 4 / 1024 * per_kib;
    if (n == 1 || ns < least) {
      least = ns;
      best = {pg, pd, (int)kpart};
    }
  }
  return best;
}

// Tiles. Hidden values: 256 x 128, or 128 x 64 where there are 512 of them (4096 tokens, d = d_ff = 1024: the call takes 175
// us instead of 192; with 256 of them no difference), or 64 x 64. dx and weight gradients: 256 x 256, or 128 x 128 where dx
// has 128 of them (2048 tokens, d = d_ff = 2048: 295 us instead of 362; 1000 tokens of 520, 40 tiles: 53 instead of 49.5),
// or 64 x 64.
bool large_tiles(int64_t T, int d, int F, bool bf16) { return bf16 && tiles(T, F, 256, 128) >= 192; }
int small_tile(const Shape& s) { return s.bf16 && tiles(s.T, s.d, 128, 128) >= 128 ? 128 : 64; }
int dx_tile(const Shape& s) { return s.bf16 && tiles(s.T, s.d, 256, 256) >= 192 ? 256 : small_tile(s); }
int weight_tile(const Shape& s, int F) { return large_tiles(s.T, s.d, F, s.bf16) ? 256 : small_tile(s); }

// Parts of dx's sum over the 2 F columns: few tokens have few tiles, each a long chain. As many as bring the workgroups to
// 320, of 512 values at least. 32 tokens, d = 2048, d_ff = 4096: the call takes 100 us instead of 128, fp32 194 instead of
// 302; with 256 tiles, 500 tokens of d = d_ff = 2048, two parts take 134 us and one 126.
int dx_parts(const Shape& s, int F) {
  if (s.T == 0 || dx_tile(s) != 64 || weight_tile(s, F) == 256) return 1;
  const int64_t wanted = 320 / tiles(s.T, s.d, 64, 64), most = 2 * F / 512;
  const int64_t parts = wanted < most ? wanted : most;
  return parts < 1 ? 1 : parts > 16 ? 16 : (int)parts;
}

template <class T, int TM, int FN, int WR, int WC>
void launch_hidden(const HiddenArgs& h, hipStream_t st) {
  hipLaunchKernelGGL((hidden_kernel<T, TM, FN, WR, WC>), dim3((unsigned)tiles(h.T, h.F, TM, FN)), dim3(64 * WR * WC), 0, st,
                     h);
}

template <class T, int WHICH>
void launch_product(int tile, const ProductArgs& g, int workgroups, hipStream_t st) {
  if constexpr (T::kSize == 2) {
    if constexpr (WHICH != (kDx | kWeights))
      if (tile == 256) {
        hipLaunchKernelGGL((product_kernel<T, 256, 256, 2, 4, WHICH>), dim3((unsigned)workgroups), dim3(512), 0, st, g);
        return;
      }
    if (tile == 128) {
      hipLaunchKernelGGL((product_kernel<T, 128, 128, 2, 4, WHICH>), dim3((unsigned)workgroups), dim3(512), 0, st, g);
      return;
    }
  }
  hipLaunchKernelGGL((product_kernel<T, 64, 64, 2, 2, WHICH>), dim3((unsigned)workgroups), dim3(256), 0, st, g);
}

template <class T>
hipError_t run(const Shape& s, int F, const uint8_t* codes, const uint8_t* scales, const void* w_gu,
               const void* w_down, const float* dy, const float* dx_in, void* dx, void* dw_gu, void* dw_down,
               char* ws, hipStream_t st) {
  constexpr bool kBf16 = T::kSize == 2;
  const int d = s.d;
  char* xb = ws;
  char* dyb = xb + up((size_t)s.T * d * T::kSize);
  char* dyl = dyb + (kBf16 ? up((size_t)s.T * d * 2) : 0);
  char* dh = dyl + (kBf16 ? up((size_t)s.T * d * 2) : 0);
  char* act = dh + up((size_t)s.T * 2 * F * T::kSize);
  char* part = act + up((size_t)s.T * F * T::kSize);
  hipError_t e;
  if (s.T > 0) {
    if (kBf16) {
      const int64_t blocks = (s.T * d / 8 + 255) / 256;
      hipLaunchKernelGGL(operands_kernel, dim3((unsigned)(blocks > 65536 ? 65536 : blocks)), dim3(256), 0, st, codes,
                         scales, dy, (uint16_t*)xb, (uint16_t*)dyb, (uint16_t*)dyl, s.T, d);
    } else if ((e = launch_checkpoint_load(s.T, d, false, codes, scales, xb, st))) {
      return e;
    }
    HiddenArgs h{xb, kBf16 ? (const void*)dyb : dy, dyl, w_gu, w_down, dh, act, s.T, d, F};
    if (kBf16 && large_tiles(s.T, d, F, true)) {
      if constexpr (kBf16) launch_hidden<T, 256, 128, 4, 2>(h, st);
    } else if (kBf16 && tiles(s.T, F, 128, 64) >= 512) {
      if constexpr (kBf16) launch_hidden<T, 128, 64, 4, 2>(h, st);
    } else {
      launch_hidden<T, 64, 64, 2, 2>(h, st);
    }
    if ((e = hipGetLastError())) return e;
  }
  const void* dyk = kBf16 ? (const void*)dyb : dy;
  ProductArgs g{};
  const int tile = weight_tile(s, F);
  const Parts z = weight_parts(s, F, tile);
  const int zx = dx_parts(s, F);
  float* const gu_part = (float*)part;
  float* const down_part = gu_part + (z.gu > 1 ? (size_t)z.gu * 2 * F * d : 0);
  float* const dx_part = down_part + (z.down > 1 ? (size_t)z.down * F * d : 0);
  int n = 0;
  if (s.T > 0) {
    const int dxt = dx_tile(s);
    n = (int)tiles(s.T, d, dxt, dxt) * zx;
    g.p[0] = {w_gu, dh, nullptr, d, 2 * (int64_t)F, s.T, d, 2 * F, (d + dxt - 1) / dxt, zx,
              (2 * F / zx + 63) / 64 * 64, 0, dx, dx_in, dx_part};
    if constexpr (kBf16)
      if (dxt == 256 || tile == 256) {
        launch_product<T, kDx>(dxt, g, n, st);
        if ((e = hipGetLastError())) return e;
        n = 0;
      }
  }
  const int n0 = (int)tiles(2 * (int64_t)F, d, tile, tile) * z.gu, n1 = (int)tiles(d, F, tile, tile) * z.down;
  g.p[1] = {xb, dh, nullptr, d, 2 * (int64_t)F, 2 * (int64_t)F, d, (int)s.T, (d + tile - 1) / tile, z.gu, z.kpart, n,
            dw_gu, nullptr, gu_part};
  g.p[2] = {act, dyk, kBf16 ? dyl : nullptr, F, d, d, F, (int)s.T, (F + tile - 1) / tile, z.down, z.kpart, n + n0,
            dw_down, nullptr, down_part};
  if (n > 0) launch_product<T, kDx | kWeights>(tile, g, n + n0 + n1, st);
  else launch_product<T, kWeights>(tile, g, n0 + n1, st);
  if ((e = hipGetLastError())) return e;
  const int64_t quads = (int64_t)F * d / 4;
  const Quads q{{zx > 1 ? s.T * d / 4 : 0, z.gu > 1 ? 2 * quads : 0, z.down > 1 ? quads : 0}};
  if (const int64_t all = q.n4[0] + q.n4[1] + q.n4[2]) {
    const int64_t blocks = (all + 255) / 256;
    hipLaunchKernelGGL(add_parts_kernel<T>, dim3((unsigned)(blocks > 65536 ? 65536 : blocks)), dim3(256), 0, st, g, q);
  }
  return hipGetLastError();
}

}  // namespace

size_t shared_backward_ws_bytes(const Shape& s, int F) {
  const size_t size = s.bf16 ? 2 : 4, T = (size_t)s.T;
  const Parts z = weight_parts(s, F, weight_tile(s, F));
  return up(T * s.d * size) + (s.bf16 ? 2 * up(T * s.d * 2) : 0) + up(T * 2 * F * size) + up(T * F * size) +
         up(((z.gu > 1 ? 2 * (size_t)z.gu : 0) + (z.down > 1 ? (size_t)z.down : 0)) * F * s.d * 4 +
            (dx_parts(s, F) > 1 ? dx_parts(s, F) * T * s.d * 4 : 0));
}

hipError_t launch_shared_backward(const Shape& s, int F, const uint8_t* codes, const uint8_t* scales,
                                  const void* w_gu, const void* w_down, const float* dy, const float* dx_in, void* dx,
                                  void* dw_gu, void* dw_down, void* ws, hipStream_t st) {
  return s.bf16 ? run<BF16>(s, F, codes, scales, w_gu, w_down, dy, dx_in, dx, dw_gu, dw_down, (char*)ws, st)
                : run<F32>(s, F, codes, scales, w_gu, w_down, dy, dx_in, dx, dw_gu, dw_down, (char*)ws, st);
}

}  // namespace omnimoe
