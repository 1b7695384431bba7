// The shared branch (Eq. 7's SwiGLU block) with low-rank adapters of many requests: token t, whose adapter is e,
//   low  = s_e A_gu[e] x               [2 r]: the first r values for the gate rows, the others for the up rows
//   g    = W_g x + B_gate[e] low[:r],  u = W_u x + B_up[e] low[r:],  a = silu(g) u
//   low' = s_e A_down[e] a             [r]
//   y    = y_in + W_down a + B_down[e] low'
//
// Up to 64 tokens (kFewTokens) every weight is read once and that bounds the call: four launches, a weight row's tile of
// all tokens beside the A rows of every adapter's tokens (sixteen tokens of one adapter to a tile), then B's rows, then
// the same for the other projection.
// More tokens are put in the order of their adapters (one workgroup counts, places and lists runs of up to sixteen
// tokens of one adapter), and the projections run as tile products whose rows follow that order. The low-rank part of a tile is
// r more values of its summed index: for every adapter among a 32-token block's rows (few, in that order) the block's low
// values meet that adapter's B rows on the matrix cores, and a token keeps the sum of its own adapter only, so that no
// value of one request reaches another's. The order of the tokens of one adapter is left to LDS atomics: no token's
// result depends on its place.
// bf16 layers round a to bf16 for the matrix cores, as omnimoe_shared_mlp does, and with more than 64 tokens low and low'
// (their expansion to few tokens is on the vector units, in fp32); sums are fp32. y, itself rounded to bf16, is 0.0019 to
// 0.0022 of its norm from the exact one; rounded once from fp32 values it is 0.0017.
#include "few_tile.hpp"
#include "internal.hpp"
#include "tile_gemm.hpp"

namespace omnimoe {
namespace {

constexpr int kFewTokens = 64;
constexpr int kMaxParts = 4;  // of a few-token projection's summed index

struct AdapterArgs {
  const void *x, *w_gu, *w_down;  // [T, d], [2 F, d], [d, F]
  const void *a_gu, *b_gu, *a_down, *b_down;
  const float* scale;  // [n], or NULL: 1
  const int32_t* ids;  // [T]
  const float* y_in;   // [T, d], or NULL
  void* y;
  int T, d, F, n, r;
  float* raw;      // few tokens: [parts, T, 2 F] W_gu x, later [parts, T, d] W_down a
  float* low;      // few tokens: [T, 2 r], later [T, r]
  void* lowt;      // in the layer's type and in sorted order: [T, 2 r], later [T, r]
  void* act;       // [T, F], in sorted order
  int32_t* order;  // [T] tokens by adapter, those without one last
  int32_t* ident;  // [T] their adapters, -1 without one
  int4* runs;      // first place, tokens, adapter of a run
  int* nruns;
};

__device__ __forceinline__ int adapter_of(const AdapterArgs& p, int t) {
  const int e = p.ids[t];
  return (unsigned)e < (unsigned)p.n ? e : -1;
}

// ---------------------------------------------------------------- up to 64 tokens

// Workgroups of the weights' rows (16 RB rows a workgroup and one of `splits` parts of the summed index, all tokens),
// then of the A rows: sixteen rows for up to sixteen tokens of one adapter, the workgroup of a token that is the first of
// such a group (others leave). TB: blocks of sixteen tokens. DOWN: the second projection.
// With many tokens it is their rows that a workgroup reads most of (64 tokens: 128 KiB for 64 KiB of weights even so);
// hence two row blocks and a part of the index instead of one block and the whole: 64 tokens, d = 2048, F = 2048: 12.0
// and 9.0 us instead of 14.6 and 12.5. With sixteen or fewer the parts cost more than they give (5.9 us instead of 5.2).
struct RowSplit {
  int weight_groups, splits, chunks, a_groups;  // chunks: 16-byte chunks of a row in a part
};
template <bool BF16, int RB, int TB, bool DOWN>
__global__ __launch_bounds__(256) void few_rows_kernel(AdapterArgs p, RowSplit split) {
  constexpr int W = 4, E = Chunk<BF16>::kElems, kSize = BF16 ? 2 : 4;
  __shared__ f32x4 tiles[W][RB * TB][64];
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int K = DOWN ? p.F : p.d, chunks = K / E;
  const char* const in = (const char*)(DOWN ? p.act : p.x);
  if ((int)blockIdx.x < split.weight_groups) {
    const int group = blockIdx.x / split.splits, part = blockIdx.x - group * split.splits;
    const int rows = DOWN ? p.d : 2 * p.F, r0 = group * 16 * RB, c0 = part * split.chunks;
    const uint4* row[RB];
    const uint4* tok[TB];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
      const int r = r0 + 16 * b + (l & 15) < rows ? r0 + 16 * b + (l & 15) : rows - 1;
      row[b] = (const uint4*)((const char*)(DOWN ? p.w_down : p.w_gu) + (int64_t)r * K * kSize) + c0;
    }
#pragma unroll
    for (int b = 0; b < TB; ++b) {
      const int t = 16 * b + (l & 15) < p.T ? 16 * b + (l & 15) : p.T - 1;
      tok[b] = (const uint4*)(in + (int64_t)t * K * kSize) + c0;
    }
    f32x4 acc[RB * TB];
    wave_tile<BF16, RB, TB, TB, W>(row, tok, chunks - c0 < split.chunks ? chunks - c0 : split.chunks, w, acc);
    add_tiles(acc, tiles, w, l);
    if (w == 0)
#pragma unroll
      for (int b = 0; b < RB; ++b) {
        const int o = r0 + 16 * b + 4 * (l >> 4);
        if (o >= rows) break;
#pragma unroll
        for (int n = 0; n < TB; ++n) {
          const int t = 16 * n + (l & 15);
          if (t < p.T) *(f32x4*)(p.raw + ((int64_t)part * p.T + t) * rows + o) = acc[b * TB + n];
        }
      }
    return;
  }
  const int g = (int)blockIdx.x - split.weight_groups, t = g / split.a_groups, rows = DOWN ? p.r : 2 * p.r;
  const int r0 = (g - t * split.a_groups) * 16;
  const int mine = l < p.T ? adapter_of(p, l) : -1;
  const int e = readlane_i32(mine, t);
  uint64_t same = __ballot(mine == e);
  if (e < 0 || __popcll(same & ((1ull << t) - 1ull)) % 16) return;
  same &= ~((1ull << t) - 1ull);
  int token = t, last = t, count = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    if (same) {
      last = __builtin_ctzll(same);
      same &= same - 1;
      ++count;
    }
    if ((l & 15) == i) token = last;
  }
  const int r = r0 + (l & 15) < rows ? r0 + (l & 15) : rows - 1;
  const uint4* const tok[1] = {(const uint4*)(in + (int64_t)token * K * kSize)};
  const uint4* const row[1] = {
      (const uint4*)((const char*)(DOWN ? p.a_down : p.a_gu) + ((int64_t)e * rows + r) * K * kSize)};
  f32x4 acc[1];
  wave_tile<BF16, 1, 1, 1, W>(row, tok, chunks, w, acc);
  f32x4(&one)[W][1][64] = *(f32x4(*)[W][1][64])tiles;
  add_tiles(acc, one, w, l);
  const int o = r0 + 4 * (l >> 4);
  if (w == 0 && (l & 15) < count && o < rows) {
    const float s = p.scale ? p.scale[e] : 1.0f;
    *(f32x4*)(p.low + (int64_t)token * rows + o) = acc[0] * s;
  }
}

// Dot of a B row (r values) with low values in LDS.
template <bool BF16>
__device__ __forceinline__ float low_dot(const void* b, int64_t row, const float* low, int r) {
  float s = 0.0f;
  for (int k = 0; k < r; k += 8) {
    if constexpr (BF16) {
      const uint4 v = *(const uint4*)((const uint16_t*)b + row * r + k);
      const uint32_t q[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s = fmaf(bf16_lo(q[i]), low[k + 2 * i], s);
        s = fmaf(bf16_hi(q[i]), low[k + 2 * i + 1], s);
      }
    } else {
      const float* const b4 = (const float*)b + row * r + k;
      const float4 v = *(const float4*)b4, u = *(const float4*)(b4 + 4);
      s = fmaf(v.x, low[k], s);
      s = fmaf(v.y, low[k + 1], s);
      s = fmaf(v.z, low[k + 2], s);
      s = fmaf(v.w, low[k + 3], s);
      s = fmaf(u.x, low[k + 4], s);
      s = fmaf(u.y, low[k + 5], s);
      s = fmaf(u.z, low[k + 6], s);
      s = fmaf(u.w, low[k + 7], s);
    }
  }
  return s;
}

__device__ __forceinline__ void store1(uint16_t* p, float v) { *p = bf16_rne(v); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }

// B's rows of one token: a value of a (or of y) a thread. 3 to 4 us each, little above a launch's own time.
template <bool BF16, bool DOWN>
__global__ __launch_bounds__(256) void few_expand_kernel(AdapterArgs p, int splits) {
  typedef typename std::conditional<BF16, uint16_t, float>::type elem;
  extern __shared__ float low[];
  const int t = blockIdx.y, e = adapter_of(p, t), width = DOWN ? p.d : p.F, rows = DOWN ? p.r : 2 * p.r;
  if (e >= 0)
    for (int k = threadIdx.x; k < rows; k += 256) low[k] = p.low[t * rows + k];
  __syncthreads();
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= width) return;
  if constexpr (DOWN) {
    float v = p.raw[(int64_t)t * p.d + c];
    for (int k = 1; k < splits; ++k) v += p.raw[((int64_t)k * p.T + t) * p.d + c];
    if (e >= 0) v += low_dot<BF16>(p.b_down, (int64_t)e * p.d + c, low, p.r);
    if (p.y_in) v += p.y_in[(int64_t)t * p.d + c];
    store1((elem*)p.y + (int64_t)t * p.d + c, v);
  } else {
    float g = 0.0f, u = 0.0f;
    for (int k = 0; k < splits; ++k) {
      const float* const raw = p.raw + ((int64_t)k * p.T + t) * 2 * p.F + c;
      g += raw[0];
      u += raw[p.F];
    }
    if (e >= 0) {
      g += low_dot<BF16>(p.b_gu, (int64_t)e * 2 * p.F + c, low, p.r);
      u += low_dot<BF16>(p.b_gu, (int64_t)e * 2 * p.F + p.F + c, low + p.r, p.r);
    }
    store1((elem*)p.act + (int64_t)t * p.F + c, activation(1, g) * u);
  }
}

// ---------------------------------------------------------------- more tokens

// Counts this lane's token into its bin: its place there. Neighbouring tokens are often of one request, so that the
// first four bins met in a wave take one LDS atomic each (4096 tokens of 16 adapters: 7.3 us; an atomic a token 10).
__device__ __forceinline__ int place_in(int* bins, int bin) {  // bin < 0: no token
  int at = 0;
  bool open = bin >= 0;
  for (int k = 0; k < 4; ++k) {
    const uint64_t todo = __ballot(open);
    if (!todo) return at;
    const int lead = __builtin_ctzll(todo), b = readlane_i32(bin, lead);
    const uint64_t same = __ballot(open && bin == b);
    int base = 0;
    if (lane_id() == lead) base = atomicAdd(bins + b, __popcll(same));
    base = readlane_i32(base, lead);
    if (open && bin == b) {
      at = base + __popcll(same & lanemask_lt());
      open = false;
    }
  }
  if (open) at = atomicAdd(bins + bin, 1);
  return at;
}

// Tokens by adapter (bin n: none), and the runs of up to kRun places of one adapter. One workgroup.
constexpr int kPlanThreads = 1024, kRun = 16;
__global__ __launch_bounds__(kPlanThreads) void plan_kernel(AdapterArgs p) {
  extern __shared__ int bins[];  // [n + 1] counts, then the next free place
  __shared__ int sums[2][kPlanThreads / 64];
  const int tid = threadIdx.x, l = tid & 63, w = tid >> 6, nb = p.n + 1;
  for (int i = tid; i < nb; i += kPlanThreads) bins[i] = 0;
  __syncthreads();
  for (int t0 = 0; t0 < p.T; t0 += kPlanThreads) {
    const int e = t0 + tid < p.T ? adapter_of(p, t0 + tid) : 0;
    place_in(bins, t0 + tid >= p.T ? -1 : e < 0 ? p.n : e);
  }
  __syncthreads();
  // A thread's bins are neighbours; exclusive sums of tokens and of runs over the threads.
  const int per = (nb + kPlanThreads - 1) / kPlanThreads, b0 = tid * per, b1 = b0 + per < nb ? b0 + per : nb;
  int tokens = 0, runs = 0;
  for (int i = b0; i < b1; ++i) {
    tokens += bins[i];
    if (i < p.n) runs += (bins[i] + kRun - 1) / kRun;
  }
  int at = wave_excl_scan_i32(tokens), run = wave_excl_scan_i32(runs);
  if (l == 63) {
    sums[0][w] = at + tokens;
    sums[1][w] = run + runs;
  }
  __syncthreads();
  for (int i = 0; i < w; ++i) {
    at += sums[0][i];
    run += sums[1][i];
  }
  if (tid == kPlanThreads - 1) *p.nruns = run + runs;
  for (int i = b0; i < b1; ++i) {
    const int count = bins[i];
    bins[i] = at;
    if (i < p.n)
      for (int k = 0; k < count; k += kRun) p.runs[run++] = make_int4(at + k, min(count - k, kRun), i, 0);
    at += count;
  }
  __syncthreads();
  for (int t0 = 0; t0 < p.T; t0 += kPlanThreads) {
    const int t = t0 + tid, e = t < p.T ? adapter_of(p, t) : 0;
    const int place = place_in(bins, t >= p.T ? -1 : e < 0 ? p.n : e);
    if (t < p.T) {
      p.order[place] = t;
      p.ident[place] = e;
    }
  }
}

// low values of a run's tokens: 16 RB rows of A a workgroup, two blocks where there are more than sixteen (4096 tokens of
// 16 adapters, d = d_ff = 2048, rank 32: 16.4 and 11.7 us instead of 19.4 and 12.4). Bound by the loads of rows from L2;
// runs of 32 and 64 tokens read less but are fewer: 20.1 and 18.0, 12.6 and 16.8 us.
template <bool BF16, int RB, bool DOWN>
__global__ __launch_bounds__(256) void run_low_kernel(AdapterArgs p) {
  constexpr int W = 4, E = Chunk<BF16>::kElems, kSize = BF16 ? 2 : 4;
  __shared__ f32x4 tiles[W][RB][64];
  if ((int)blockIdx.x >= *p.nruns) return;
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int4 run = p.runs[blockIdx.x];
  const int rows = DOWN ? p.r : 2 * p.r, K = DOWN ? p.F : p.d, r0 = blockIdx.y * 16 * RB;
  const int place = run.x + ((l & 15) < run.y ? (l & 15) : run.y - 1);
  const uint4* const tok[1] = {(const uint4*)(DOWN ? (const char*)p.act + (int64_t)place * K * kSize
                                                   : (const char*)p.x + (int64_t)p.order[place] * K * kSize)};
  const uint4* row[RB];
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const int r = r0 + 16 * b + (l & 15) < rows ? r0 + 16 * b + (l & 15) : rows - 1;
    row[b] = (const uint4*)((const char*)(DOWN ? p.a_down : p.a_gu) + ((int64_t)run.z * rows + r) * K * kSize);
  }
  f32x4 acc[RB];
  wave_tile<BF16, RB, 1, 1, W>(row, tok, K / E, w, acc);
  add_tiles(acc, tiles, w, l);
  if (w || (l & 15) >= run.y) return;
  const float s = p.scale ? p.scale[run.z] : 1.0f;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const int o = r0 + 16 * b + 4 * (l >> 4);
    if (o >= rows) break;
    typedef typename std::conditional<BF16, uint16_t, float>::type elem;
    store4((elem*)p.lowt + (int64_t)place * rows + o, acc[b][0] * s, acc[b][1] * s, acc[b][2] * s, acc[b][3] * s);
  }
}

// Sixteen bytes of k values 16 ks + 8 half (bf16) or 8 ks + 4 half (fp32) of a row of r values, zeros past its end.
template <class T>
__device__ __forceinline__ typename T::frag low_frag(const typename T::elem* row, int r, int ks, int half) {
  constexpr int kPer = 16 / T::kSize;
  const int k = (2 * ks + half) * kPer;
  const uint4 v = *(const uint4*)(row + (k < r ? k : 0));
  return __builtin_bit_cast(typename T::frag, k < r ? v : make_uint4(0, 0, 0, 0));
}

// A tile of TM places x TN weight rows: of W_gu TN / 2 gate and TN / 2 up rows (DOWN: of W_down TN), then the low-rank
// part, then a = silu(g) u by places (DOWN: y by tokens). A wave of W_gu's tile holds gate rows and the same features' up
// rows; where it has one block only (kApart), the second half of the waves holds the up rows and hands them over in LDS.
// Bound as the tile products are: 4096 tokens, d = d_ff = 2048, rank 32, 16 adapters: 79 and 63 us, 0.87 and 0.55 PFLOP/s
// (the down projection has half the tiles).
template <class T, int TM, int TN, int WR, int WC, bool DOWN>
__global__ __launch_bounds__(64 * WR * WC) void adapter_tile_kernel(AdapterArgs p) {
  constexpr int NW = WR * WC, MJ = TM / WR / 32, NI = TN / WC / 32, FN = TN / 2;
  constexpr bool kApart = !DOWN && NI == 1;
  static_assert(DOWN || NI % 2 == 0 || (MJ == 1 && WR == 1 && WC % 2 == 0), "gate rows and their up rows");
  typedef typename T::elem elem;
  __shared__ __attribute__((aligned(1024))) unsigned char st0[(TM + TN) * 128], st1[(TM + TN) * 128];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wid / WC, wc = wid % WC;
  const int K = DOWN ? p.F : p.d, width = DOWN ? p.d : p.F, step = DOWN ? TN : FN, tiles_n = (width + step - 1) / step;
  const int m0 = (int)(blockIdx.x / (unsigned)tiles_n) * TM, n0 = (int)(blockIdx.x % (unsigned)tiles_n) * step;
  int a0[NI], b0[MJ], c0[NI];  // c0: the block's first output column
#pragma unroll
  for (int j = 0; j < MJ; ++j) b0[j] = (wr * MJ + j) * 32;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    if constexpr (DOWN || kApart) {
      a0[i] = (wc * NI + i) * 32;
      c0[i] = n0 + (kApart ? a0[i] % FN : a0[i]);
    } else {  // even blocks: gate rows, odd ones: the same features' up rows
      const int f = (wc * (NI / 2) + i / 2) * 32;
      a0[i] = f + (i & 1) * FN;
      c0[i] = n0 + f;
    }
  }
  tg_f32x16 acc[NI][MJ];
  tile_zero(acc);
  {
    TileOperand<T, TN, false, NW> a;
    TileOperand<T, TM, false, NW> b;
    a.init((const elem*)(DOWN ? p.w_down : p.w_gu), K, wid, lane, [&](int r) {
      if constexpr (DOWN) return n0 + r < width ? n0 + r : width - 1;
      const int f = n0 + (r < FN ? r : r - FN);
      return (f < width ? f : width - 1) + (r < FN ? 0 : width);
    });
    // (the hidden values of a pass may take more than 4 GiB: their rows are counted from the tile's first)
    b.init(DOWN ? (const elem*)p.act + (int64_t)m0 * K : (const elem*)p.x, K, wid, lane, [&](int r) {
      const int place = m0 + r < p.T ? m0 + r : p.T - 1;
      return DOWN ? place - m0 : p.order[place];
    });
    const TileRange all[2] = {{K, 0, 0}, {0, 0, 0}};
    tile_sum<T>(a, b, all, a0, b0, st0, st1, wid, lane, acc);
  }
  const int half = lane >> 5, r = p.r, ld = DOWN ? r : 2 * r, steps = (r * T::kSize + 31) / 32;
#pragma unroll
  for (int j = 0; j < MJ; ++j) {
    const int place = m0 + b0[j] + (lane & 31);
    const int e = place < p.T ? p.ident[place] : -1;
    const elem* const low = (const elem*)p.lowt + (int64_t)(place < p.T ? place : p.T - 1) * ld;
    for (uint64_t todo = __ballot(e >= 0); todo;) {
      const int f = readlane_i32(e, __builtin_ctzll(todo));
      todo &= ~__ballot(e == f);
      const elem* const b = (const elem*)(DOWN ? p.b_down : p.b_gu) + (int64_t)f * (DOWN ? p.d : 2 * p.F) * r;
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const int up = kApart ? wc >= WC / 2 : !DOWN && (i & 1), c = c0[i] + (lane & 31);
        const elem* const brow = b + (int64_t)((c < width ? c : width - 1) + (up ? p.F : 0)) * r;
        tg_f32x16 s;
#pragma unroll
        for (int q = 0; q < 16; ++q) s[q] = 0.f;
        for (int ks = 0; ks < steps; ++ks)
          tile_mma(s, low_frag<T>(brow, r, ks, half), low_frag<T>(low + (up ? r : 0), r, ks, half));
#pragma unroll
        for (int q = 0; q < 16; ++q) acc[i][j][q] += e == f ? s[q] : 0.0f;
      }
    }
    tg_f32x16 ups;
    if constexpr (kApart) {
      float4(*const turned)[4][64] = (float4(*)[4][64])st0;
      __syncthreads();
      if (wc >= WC / 2)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          turned[wc - WC / 2][q][lane] =
              make_float4(acc[0][j][4 * q], acc[0][j][4 * q + 1], acc[0][j][4 * q + 2], acc[0][j][4 * q + 3]);
      __syncthreads();
      if (wc >= WC / 2) return;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float4 v = turned[wc][q][lane];
        ups[4 * q] = v.x;
        ups[4 * q + 1] = v.y;
        ups[4 * q + 2] = v.z;
        ups[4 * q + 3] = v.w;
      }
    }
    if (place >= p.T) continue;
    if constexpr (DOWN) {
      const int64_t at = (int64_t)p.order[place] * p.d;
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int c = c0[i] + 8 * q + 4 * half;
          if (c >= width) continue;
          float4 v = make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
          if (p.y_in) {
            const float4 y = *(const float4*)(p.y_in + at + c);
            v.x += y.x;
            v.y += y.y;
            v.z += y.z;
            v.w += y.w;
          }
          store4((elem*)p.y + at + c, v.x, v.y, v.z, v.w);
        }
    } else {
#pragma unroll
      for (int i = 0; i < NI; i += 2)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int c = c0[i] + 8 * q + 4 * half;
          if (c >= width) continue;
          float v[4];
#pragma unroll
          for (int k = 0; k < 4; ++k)
            v[k] = activation(1, acc[i][j][4 * q + k]) * (kApart ? ups[4 * q + k] : acc[kApart ? 0 : i + 1][j][4 * q + k]);
          store4((elem*)p.act + (int64_t)place * p.F + c, v[0], v[1], v[2], v[3]);
        }
    }
  }
}

size_t up(size_t v) { return (v + 255) & ~(size_t)255; }

// Tokens of one pass: its tiles' offsets count over all their rows of x.
constexpr int64_t kPassTokens = 65536;
static_assert(kPassTokens * kMaxWidth * 2 < kTileReach && kPassTokens * kMaxWidthF32 * 4 < kTileReach, "rows of x");

struct Layout {
  size_t raw, low, lowt, act, order, ident, runs, bytes;
  int64_t max_runs;
};
Layout layout(const Shape& s, int F, int n, int r) {
  const size_t size = s.bf16 ? 2 : 4, T = (size_t)(s.T < kPassTokens ? s.T : kPassTokens);
  Layout o{};
  size_t at = 256;  // the runs' number
  auto take = [&](size_t bytes) {
    const size_t v = at;
    at += up(bytes);
    return v;
  };
  o.act = take(T * F * size);
  if (s.T <= kFewTokens) {
    o.raw = take(kMaxParts * T * (2 * (size_t)F > (size_t)s.d ? 2 * (size_t)F : (size_t)s.d) * 4);
    o.low = take(T * 2 * r * 4);
  } else {
    o.max_runs = (int64_t)(T / kRun + (T < (size_t)n ? T : (size_t)n));
    o.lowt = take(T * 2 * r * size);
    o.order = take(T * 4);
    o.ident = take(T * 4);
    o.runs = take((size_t)o.max_runs * 16);
  }
  o.bytes = at;
  return o;
}

// Parts of a few-token projection with more than sixteen tokens: of at least 512 bytes a row, as many as bring the
// weights' workgroups to one per compute unit, four at most.
RowSplit row_split(int rows, int K, int size, int rb, int a_groups) {
  RowSplit o;
  const int groups = (rows + 16 * rb - 1) / (16 * rb), chunks = K * size / 16;
  int parts = 1;
  while (rb > 1 && parts < kMaxParts && groups * parts < 256 && chunks / (2 * parts) >= 32) parts *= 2;
  o.chunks = ((chunks + parts - 1) / parts + 7) / 8 * 8;
  o.splits = (chunks + o.chunks - 1) / o.chunks;
  o.weight_groups = groups * o.splits;
  o.a_groups = a_groups;
  return o;
}

template <bool BF16, bool DOWN>
int launch_rows(const AdapterArgs& p, hipStream_t st) {
  const int tb = (p.T + 15) / 16, rb = tb > 1 ? 2 : 1;
  const RowSplit split = row_split(DOWN ? p.d : 2 * p.F, DOWN ? p.F : p.d, BF16 ? 2 : 4, rb,
                                   p.n ? ((DOWN ? p.r : 2 * p.r) + 15) / 16 : 0);
  const dim3 grid((unsigned)(split.weight_groups + p.T * split.a_groups));
#define OMNIMOE_ROWS(RB_, TB_) \
  hipLaunchKernelGGL((few_rows_kernel<BF16, RB_, TB_, DOWN>), grid, dim3(256), 0, st, p, split)
  if (tb == 1) OMNIMOE_ROWS(1, 1);
  else if (tb == 2) OMNIMOE_ROWS(2, 2);
  else if (tb == 3) OMNIMOE_ROWS(2, 3);
  else OMNIMOE_ROWS(2, 4);
#undef OMNIMOE_ROWS
  return split.splits;
}

template <bool BF16, bool DOWN>
void launch_low(const AdapterArgs& p, int64_t max_runs, hipStream_t st) {
  const int rows = DOWN ? p.r : 2 * p.r;
  if (rows > 16)
    hipLaunchKernelGGL((run_low_kernel<BF16, 2, DOWN>), dim3((unsigned)max_runs, (unsigned)((rows + 31) / 32)), dim3(256),
                       0, st, p);
  else
    hipLaunchKernelGGL((run_low_kernel<BF16, 1, DOWN>), dim3((unsigned)max_runs), dim3(256), 0, st, p);
}

// The largest tile that leaves few compute units without one: a 4096-token batch, d = d_ff = 2048, down projection (128
// tiles of 256 x 256) 68 us on 64 x 128, 65 on 128 x 256; fp32, 333 tokens, 520 wide: 30 and 31 us on 64 x 128 (54 and 30
// tiles), 20 and 20 on 32 x 128.
template <class T, int TM, int TN, int WR, int WC, bool DOWN>
bool try_tile(const AdapterArgs& p, int64_t least, hipStream_t st) {
  const int64_t width = DOWN ? p.d : p.F, step = DOWN ? TN : TN / 2;
  const int64_t tiles = ((int64_t)p.T + TM - 1) / TM * ((width + step - 1) / step);
  if (tiles < least) return false;
  hipLaunchKernelGGL((adapter_tile_kernel<T, TM, TN, WR, WC, DOWN>), dim3((unsigned)tiles), dim3(64 * WR * WC), 0, st, p);
  return true;
}
template <class T, bool DOWN>
void launch_tiles(const AdapterArgs& p, hipStream_t st) {
  if constexpr (T::kSize == 2) {
    if (try_tile<T, 256, 256, 2, 4, DOWN>(p, 192, st)) return;
    if (try_tile<T, 128, 256, 2, 4, DOWN>(p, 192, st)) return;
  }
  if (try_tile<T, 64, 128, 2, 2, DOWN>(p, 192, st)) return;
  try_tile<T, 32, 128, 1, 4, DOWN>(p, 0, st);
}

template <class T>
hipError_t run(const AdapterArgs& p, const Layout& o, bool few, hipStream_t st) {
  constexpr bool kBf16 = T::kSize == 2;
  hipError_t e;
  if (few) {
    const unsigned T_ = (unsigned)p.T;
    const int parts = launch_rows<kBf16, false>(p, st);
    hipLaunchKernelGGL((few_expand_kernel<kBf16, false>), dim3((unsigned)((p.F + 255) / 256), T_), dim3(256),
                       (size_t)2 * p.r * 4, st, p, parts);
    if ((e = hipGetLastError())) return e;
    const int down_parts = launch_rows<kBf16, true>(p, st);
    hipLaunchKernelGGL((few_expand_kernel<kBf16, true>), dim3((unsigned)((p.d + 255) / 256), T_), dim3(256),
                       (size_t)p.r * 4, st, p, down_parts);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(plan_kernel, dim3(1), dim3(kPlanThreads), (size_t)(p.n + 1) * 4, st, p);
  if (p.n) launch_low<kBf16, false>(p, o.max_runs, st);
  if ((e = hipGetLastError())) return e;
  launch_tiles<T, false>(p, st);
  if (p.n) launch_low<kBf16, true>(p, o.max_runs, st);
  if ((e = hipGetLastError())) return e;
  launch_tiles<T, true>(p, st);
  return hipGetLastError();
}

}  // namespace

size_t adapters_ws_bytes(const Shape& s, int F, int n, int r) { return layout(s, F, n, r).bytes; }

hipError_t launch_adapters(const Shape& s, int F, const AdapterTables& t, const void* x, const void* w_gu,
                           const void* w_down, const int32_t* ids, const float* y_in, void* y, void* ws,
                           hipStream_t st) {
  const Layout o = layout(s, F, t.n, t.rank);
  const size_t size = s.bf16 ? 2 : 4;
  char* w = (char*)ws;
  AdapterArgs p;
  p.w_gu = w_gu;
  p.w_down = w_down;
  p.a_gu = t.a_gu;
  p.b_gu = t.b_gu;
  p.a_down = t.a_down;
  p.b_down = t.b_down;
  p.scale = t.scale;
  p.d = s.d;
  p.F = F;
  p.n = t.n;
  p.r = t.rank;
  p.raw = (float*)(w + o.raw);
  p.low = (float*)(w + o.low);
  p.lowt = w + o.lowt;
  p.act = w + o.act;
  p.order = (int32_t*)(w + o.order);
  p.ident = (int32_t*)(w + o.ident);
  p.runs = (int4*)(w + o.runs);
  p.nruns = (int*)w;
  for (int64_t t0 = 0; t0 < s.T; t0 += kPassTokens) {
    p.T = (int)(s.T - t0 < kPassTokens ? s.T - t0 : kPassTokens);
    p.x = (const char*)x + (size_t)t0 * s.d * size;
    p.ids = ids + t0;
    p.y_in = y_in ? y_in + t0 * s.d : nullptr;
    p.y = (char*)y + (size_t)t0 * s.d * size;
    const bool few = s.T <= kFewTokens;  // (as the workspace is laid out)
    const hipError_t e = s.bf16 ? run<BF16>(p, o, few, st) : run<F32>(p, o, few, st);
    if (e) return e;
  }
  return hipSuccess;
}

}  // namespace omnimoe
