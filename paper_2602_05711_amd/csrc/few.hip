// The whole feed-forward layer (Eq. 7: routed and shared branch) for up to sixteen tokens in two kernels.
//
//   few_products  every product that needs only x: the row and column logits (Eq. 9) and the shared branch's hidden
//                 values a = silu(W_g x) (.) (W_u x). Reading the sub-keys and W_g, W_u once is its cost.
//   few_finish    a workgroup per (token, head) selects (Eq. 11, 1, 2), forms g act(x . u) of its K picks and adds their
//                 a v rows; further workgroups form the down projection of all tokens beside it. Whoever finishes a
//                 range of a token's columns last (a counter) adds the heads' partial rows there, in order, then the
//                 shared branch's.
//
// The partial rows and the counters cross XCDs inside one kernel, whose L2s are not coherent with each other: partial
// rows are stored and loaded at agent scope (past L2), every thread waits for its stores (vmcnt) before the barrier
// behind which one wave counts the workgroup in, and nothing waits for another workgroup.
#include <type_traits>

#include "bf16_parts.hpp"
#include "cand_table.hpp"
#include "few_tile.hpp"
#include "internal.hpp"

namespace omnimoe {
namespace {

constexpr int kTokens = 16;
constexpr int kSplit = 3;  // bf16 values of a hidden value
// The columns are divided into at most 64 ranges of 128. The workgroups of the down projection (eight to a range, sixteen
// columns each) count themselves into their range, whose last one counts it in for every token; a head's counts in for
// each range of its token. With a single range a workgroup of the down projection that came last would have all the tokens
// to add: 16 tokens, d = d_ff = 2048, back to back, 52.5 us a call instead of 27.7 (ranges of 256 columns 29.4, of 64 27.4).
// Without a shared branch there is one range, all the columns.
constexpr int kRanges = 64, kRangeGroups = 8;
static_assert(kRanges * kRangeGroups * 16 >= kMaxWidth, "a range for every column");
constexpr int kRangeLine = 16;                                       // (counters of different ranges lie 64 bytes apart)
constexpr int kCounts = kTokens * kRanges + kRanges * kRangeLine;    // the tokens' by ranges, then the ranges'

struct FewArgs {
  const void *x, *keys[2], *u, *v, *w_gu, *w_down;
  float* y;
  int32_t* idx;   // or NULL
  float* gates;   // or NULL
  float* logits;  // [T H, npad[0] + npad[1]]
  void* act;      // bf16: [kSplit][kTokens, F]; fp32: [kTokens, F]
  float* part;    // [T H, d] the heads' sums
  float* shared;  // [down_groups, T, 16] the down projection
  int* count;     // [kCounts]
  int T, d, F, H, K, act_kind, dk, col0;
  int n[2], npad[2];
  int key_groups[2];  // workgroups of sixteen sub-keys per half
  int down_groups;    // workgroups of sixteen output columns
  int ranges, span;   // of the columns, and the columns of one
};

// Sixteen sub-keys or eight features (their gate and up rows) a workgroup, its four waves each a quarter of k. Bound by
// the load latency of a workgroup's one pass over its rows, 48 MB in all: d = 2048, 1024 + 1024 sub-keys, 8 heads, d_ff =
// 2048: 10.1 us for one token, 13.5 for sixteen (whose rows every workgroup reads, 64 KiB from L2). Eight or sixteen waves
// took 16.8 and 18.1 us, 32 rows a workgroup 15.5.
template <bool BF16>
__global__ __launch_bounds__(256) void few_products(FewArgs p) {
  constexpr int W = 4, E = Chunk<BF16>::kElems, kSize = BF16 ? 2 : 4;
  __shared__ f32x4 tiles[W][1][64];
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6, t = l & 15;
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < kCounts / 4; i += 256) ((int4*)p.count)[i] = make_int4(0, 0, 0, 0);
  const char* const x = (const char*)p.x + (int64_t)(t < p.T ? t : p.T - 1) * p.d * kSize;
  f32x4 acc[1];
  int g = blockIdx.x;
  const int half = g < p.key_groups[0] ? 0 : 1;
  if (half) g -= p.key_groups[0];
  if (g < (half ? p.key_groups[1] : p.key_groups[0])) {
    const int n = half ? p.n[1] : p.n[0], rows = p.H * n, r0 = g * 16, r = r0 + t < rows ? r0 + t : rows - 1;
    const uint4* const row[1] = {
        (const uint4*)((const char*)(half ? p.keys[1] : p.keys[0]) + (int64_t)r * p.dk * kSize)};
    const uint4* const tok[1] = {(const uint4*)(x + (half ? p.col0 * kSize : 0))};
    wave_tile<BF16, 1, 1, 1, W>(row, tok, p.dk / E, w, acc);
    add_tiles(acc, tiles, w, l);
    if (w == 0 && t < p.T)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int key = r0 + 4 * (l >> 4) + q;
        if (key >= rows) break;
        const int h = key / n, i = key - h * n;
        p.logits[((int64_t)t * p.H + h) * (p.npad[0] + p.npad[1]) + (half ? p.npad[0] : 0) + i] = acc[0][q];
      }
    return;
  }
  // eight features a workgroup: a lane's four accumulators are the gate and up values of two of them
  const int f0 = (g - p.key_groups[1]) * 8, f = f0 + 2 * (t >> 2) + (t & 1);
  const int r = (f < p.F ? f : p.F - 1) + (t & 2 ? p.F : 0);
  const uint4* const row[1] = {(const uint4*)((const char*)p.w_gu + (int64_t)r * p.d * kSize)};
  const uint4* const tok[1] = {(const uint4*)x};
  wave_tile<BF16, 1, 1, 1, W>(row, tok, p.d / E, w, acc);
  add_tiles(acc, tiles, w, l);
  const int fo = f0 + 2 * (l >> 4);
  if (w == 0 && fo < p.F) {
    const float a0 = activation(1, acc[0][0]) * acc[0][2], a1 = activation(1, acc[0][1]) * acc[0][3];
    if constexpr (BF16) {
      // three bf16 values a feature, their sum a itself: the down projection keeps fp32's accuracy
      float r0 = a0, r1 = a1;
#pragma unroll
      for (int n = 0; n < kSplit; ++n) {
        const uint32_t h0 = bf16_part(r0), h1 = bf16_part(r1);
        *(uint32_t*)((uint16_t*)p.act + (n * kTokens + t) * p.F + fo) = h0 | (h1 << 16);
      }
    } else {
      *(float2*)((float*)p.act + t * p.F + fo) = make_float2(a0, a1);
    }
  }
}

// ---------------------------------------------------------------- few_finish

__device__ __forceinline__ void store_agent(float* p, float a, float b) {
  __hip_atomic_store((uint64_t*)p, ((uint64_t)__float_as_uint(b) << 32) | __float_as_uint(a), __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float4 load_agent4(const float* p) {
  const uint64_t a = __hip_atomic_load((const uint64_t*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  const uint64_t b = __hip_atomic_load((const uint64_t*)(p + 2), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float4(__uint_as_float((uint32_t)a), __uint_as_float((uint32_t)(a >> 32)), __uint_as_float((uint32_t)b),
                     __uint_as_float((uint32_t)(b >> 32)));
}

constexpr int kThreads = 512, kWaves = 8;

// This wave's half of a row: its best kh of n logits, best first (logit descending, index ascending), as keys (value
// order high, ~index low) in out[0 .. kh). The logits that reach a threshold that at least kh of them reach (the kh-th
// largest of the lanes' maxima, its low bits cleared) are ranked by counting; more than 64 of them are taken one after the
// other instead. That is so with ties, and with most rows for kh near 64, where the threshold is near the least of the 64
// maxima: of Gaussian logits (n = 320 to 4096) in no row for kh = 32, in 15 to 36% of them for 40, in 71 to 86% for 44, in
// nearly all from 48 on; with fewer than 4 kh logits, where fewer than kh lanes hold any, always if n > 64. One at a time
// costs most of the kernel's time: one token, 8 heads of 1024 + 1024 logits, K = 64, 61 us (K = 16: 12), one head of
// 320 + 320 49 us.
template <int R>
__device__ __forceinline__ void half_best(const float* __restrict__ logits, int n, int kh, uint64_t* __restrict__ cand,
                                          uint64_t* __restrict__ out) {
  const int l = lane_id();
  uint32_t o[R];
  uint32_t most = 0u;
#pragma unroll
  for (int c = 0; c < R / 4; ++c) {
    const float4 v = *(const float4*)(logits + 256 * c + 4 * l < logits + n ? logits + 256 * c + 4 * l : logits);
    const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) o[4 * c + q] = 256 * c + 4 * l + q < n ? ord_f32(e[q]) : 0u;
  }
#pragma unroll
  for (int k = 0; k < R; ++k) most = o[k] > most ? o[k] : most;
  uint32_t th = 0u;
#pragma unroll
  for (int b = 31; b >= 8; --b) {
    const uint32_t c = th | (1u << b);
    if (__popcll(__ballot(most >= c)) >= kh) th = c;
  }
  auto index = [&](int k) { return 256 * (k >> 2) + 4 * l + (k & 3); };
  auto key = [&](int k) { return ((uint64_t)o[k] << 32) | (0xFFFFFFFFu - (uint32_t)index(k)); };
  int total = 0;
#pragma unroll
  for (int k = 0; k < R; ++k) {
    const bool in = o[k] >= th && index(k) < n;
    const uint64_t m = __ballot(in);
    const int at = total + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32),
                                                          __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
    if (in && at < 64) cand[at] = key(k);
    total += __popcll(m);
  }
  if (l >= total) cand[l] = 0ull;
  wave_lds_sync();
  if (total <= 64) {
    const uint64_t mine = cand[l];
    int rank = 0;
    for (int j = 0; j < total; j += 8) {
      ulonglong2 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = *(const ulonglong2*)(cand + j + 2 * i);
#pragma unroll
      for (int i = 0; i < 4; ++i) rank += (v[i].x > mine ? 1 : 0) + (v[i].y > mine ? 1 : 0);
    }
    if (l < total && rank < kh) out[rank] = mine;
  } else {
    uint64_t last = ~0ull;
    for (int j = 0; j < kh; ++j) {
      uint64_t m = 0ull;
#pragma unroll
      for (int k = 0; k < R; ++k) {
        const uint64_t v = index(k) < n ? key(k) : 0ull;
        m = v < last && v > m ? v : m;
      }
#pragma unroll
      for (int b = 32; b >= 1; b >>= 1) {
        const uint64_t v = shfl_xor_u64(m, b);
        m = v > m ? v : m;
      }
      if (l == 0) out[j] = m;
      last = m;
    }
  }
}

// Tiles of a down projection: the hidden values' leading parts, and (bf16) their other parts.
template <bool BF16>
constexpr int kDownTiles = BF16 ? 2 : 1;

constexpr int kCells = 288;  // at least the 280 cells of K = 64, and what the last wave's share runs past them
struct FinishShared {
  union {
    f32x4 tiles[kWaves * kDownTiles<true>][64];
    struct {
      uint64_t cand[2][64], best[2][64];
      uint4 cell[kCells];  // score (order map of the double), id
      int rank[kCells];
      uint64_t pick_score[64];
      uint32_t pick_id[64];
      float a[64];
    };
  };
  int items, item[64];
};

__device__ __forceinline__ int count_in(int* count) {
  return __hip_atomic_fetch_add(count, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Counts the workgroup in for token t and range r of this lane of wave 0 (some lanes' only: `on`) and lists the lanes that
// were the last there; the others' stores have arrived then.
__device__ __forceinline__ void list_finished(const FewArgs& p, FinishShared& sh, bool on, int t, int r) {
  const bool last = on && count_in(p.count + t * kRanges + r) == p.H + (p.F ? 1 : 0) - 1;
  const uint64_t m = __ballot(last);
  if (last) sh.item[__popcll(m & lanemask_lt())] = lane_id();
  if (lane_id() == 0) sh.items = __popcll(m);
}

// y from the heads' sums and the down projection's, by the whole workgroup: the listed ranges of token t, or (t < 0) range
// r of the listed tokens.
__device__ __forceinline__ void add_finished(const FewArgs& p, const FinishShared& sh, int t, int r) {
  const int per = p.span / 4;
  for (int q = threadIdx.x; q < sh.items * per; q += kThreads) {
    const int n = q / per, item = sh.item[n], tok = t < 0 ? item : t;
    const int c = (t < 0 ? r : item) * p.span + (q - n * per) * 4;
    if (c >= p.d) continue;
    const float* part = p.part + (int64_t)tok * p.H * p.d + c;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f), shared = s;
    if (p.F) shared = load_agent4(p.shared + ((int64_t)(c >> 4) * p.T + tok) * 16 + (c & 15));
    for (int h0 = 0; h0 < p.H; h0 += 8) {
      float4 v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (h0 + i < p.H) v[i] = load_agent4(part + (int64_t)(h0 + i) * p.d);
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (h0 + i < p.H) {
          s.x += v[i].x;
          s.y += v[i].y;
          s.z += v[i].z;
          s.w += v[i].w;
        }
    }
    if (p.F) {
      s.x += shared.x;
      s.y += shared.y;
      s.z += shared.z;
      s.w += shared.w;
    }
    *(float4*)(p.y + (int64_t)tok * p.d + c) = s;
  }
}

template <bool BF16>
__device__ __forceinline__ void down_group(const FewArgs& p, FinishShared& sh, int g) {
  constexpr int E = Chunk<BF16>::kElems, kSize = BF16 ? 2 : 4, NB = BF16 ? kSplit : 1, NACC = kDownTiles<BF16>;
  const int l = threadIdx.x & 63, w = threadIdx.x >> 6, t = l & 15;
  const int col = g * 16 + t < p.d ? g * 16 + t : p.d - 1;
  const uint4* const row[1] = {(const uint4*)((const char*)p.w_down + (int64_t)col * p.F * kSize)};
  // (the hidden values of lanes past the last token are that token's again)
  auto act = [&](int n) { return (const uint4*)((const char*)p.act + (int64_t)(n * kTokens + t) * p.F * kSize); };
  f32x4 acc[NACC];
  if constexpr (BF16) {
    const uint4* const tok[NB] = {act(0), act(1), act(2)};
    wave_tile<BF16, 1, NB, NACC, kWaves>(row, tok, p.F / E, w, acc);
  } else {
    const uint4* const tok[NB] = {act(0)};
    wave_tile<BF16, 1, NB, NACC, kWaves>(row, tok, p.F / E, w, acc);
  }
  add_tiles(acc, *(f32x4(*)[kWaves][NACC][64])sh.tiles, w, l);
  // An infinite weight: the leading parts' sum is the infinity, or NaN where a is zero; of the others' products one may be
  // an infinity of the other sign, or zero times it.
  if constexpr (BF16)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if ((__float_as_uint(acc[0][q]) & 0x7F800000u) != 0x7F800000u) acc[0][q] += acc[1][q];
  const int r = g / kRangeGroups;
  if (w == 0) {
    // through LDS, so that a store covers whole lines: token by token, sixteen columns each
    float2* const turned = (float2*)sh.tiles;
    turned[t * 8 + 2 * (l >> 4)] = make_float2(acc[0][0], acc[0][1]);
    turned[t * 8 + 2 * (l >> 4) + 1] = make_float2(acc[0][2], acc[0][3]);
    wave_lds_sync();
    float* const o = p.shared + (int64_t)g * p.T * 16;
    for (int i = l; i < p.T * 8; i += 64) {
      const float2 v = turned[i];
      store_agent(o + 2 * i, v.x, v.y);
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): the wave's stores are past L2
    __builtin_amdgcn_fence(__ATOMIC_SEQ_CST, "workgroup");
    const int rest = p.down_groups - r * kRangeGroups;
    int last = 0;
    if (l == 0) last = count_in(p.count + kTokens * kRanges + r * kRangeLine) == min(rest, kRangeGroups) - 1;
    last = readlane_i32(last, 0);
    list_finished(p, sh, last && l < p.T, l, r);
  }
  __syncthreads();
  add_finished(p, sh, -1, r);
}

// R: logits of a half per lane. A chain of dependent steps that only the size of a step's loads can shorten (one token, K =
// 16, 8 heads, 1024 logits a half, cycles: logits 4100, threshold and survivors 2000, ranks and cells 2300, the u rows and
// dots 5900, the v rows 1800, stores and counting 1900): 12.3 us for one token, 14.0 for sixteen, 9.0 for seven of a small
// fp32 layer. For large K see half_best.
template <bool BF16, int R>
__global__ __launch_bounds__(kThreads) void few_finish(FewArgs p) {
  __shared__ FinishShared sh;
  if ((int)blockIdx.x >= p.T * p.H) {
    down_group<BF16>(p, sh, (int)blockIdx.x - p.T * p.H);
    return;
  }
  constexpr int E = Chunk<BF16>::kElems, kSize = BF16 ? 2 : 4;
  const int row = blockIdx.x, t = row / p.H, K = p.K;
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kr = K < p.n[0] ? K : p.n[0], kc = K < p.n[1] ? K : p.n[1];
  // The candidate cells (a, b), (a + 1)(b + 1) <= K: at most 280, one a thread.
  const int first = kCand.first[K], cells = kCand.first[K + 1] - first;
  const int ab = kCand.cell[first + ((int)threadIdx.x < cells ? threadIdx.x : 0)];
  if (w < 2)
    half_best<R>(p.logits + (int64_t)row * (p.npad[0] + p.npad[1]) + (w ? p.npad[0] : 0), w ? p.n[1] : p.n[0],
                 w ? kc : kr, sh.cand[w], sh.best[w]);
  __syncthreads();
  if (threadIdx.x < kCells) {
    const int a = ab >> 8, b = ab & 0xFF;
    uint64_t score = 0ull;  // (no cell: below every score)
    uint32_t id = 0xFFFFFFFFu;
    if ((int)threadIdx.x < cells && a < kr && b < kc) {
      const uint64_t ka = sh.best[0][a], kb = sh.best[1][b];
      score = ord_f64((double)f32_from_ord((uint32_t)(ka >> 32)) + (double)f32_from_ord((uint32_t)(kb >> 32)));
      id = (0xFFFFFFFFu - (uint32_t)ka) * (uint32_t)p.n[1] + (0xFFFFFFFFu - (uint32_t)kb);
    }
    sh.cell[threadIdx.x] = make_uint4((uint32_t)score, (uint32_t)(score >> 32), id, 0u);
    sh.rank[threadIdx.x] = 0;
  }
  __syncthreads();
  // Their ranks by counting (score descending, id ascending): a lane has a cell, a wave an eighth of those that it is
  // compared with. (On one wave the 50 cells of K = 16 took 6600 of the kernel's 27000 cycles.)
  const int share = (cells + kWaves - 1) / kWaves;
  for (int c = l; c < cells; c += 64) {
    const uint4 m = sh.cell[c];
    const uint64_t mine = ((uint64_t)m.y << 32) | m.x;
    int rank = 0;
    for (int j0 = w * share; j0 < (w + 1) * share; j0 += 4) {
      uint4 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = sh.cell[j0 + i];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint64_t s = ((uint64_t)v[i].y << 32) | v[i].x;
        const bool above = (s > mine) | ((s == mine) & (v[i].z < m.z));
        rank += above & (j0 + i < (w + 1) * share) ? 1 : 0;
      }
    }
    atomicAdd(&sh.rank[c], rank);
  }
  __syncthreads();
  if ((int)threadIdx.x < cells) {
    const uint4 m = sh.cell[threadIdx.x];
    const int rank = sh.rank[threadIdx.x];
    if (m.z != 0xFFFFFFFFu && rank < K) {
      sh.pick_score[rank] = ((uint64_t)m.y << 32) | m.x;
      sh.pick_id[rank] = m.z;
    }
  }
  __syncthreads();
  const uint32_t eid = sh.pick_id[l < K ? l : 0];  // lane k: pick k's expert
  // x . u of picks w, w + 8, ..., two at a time; the first v rows are requested right after the first u rows.
  // (Loads are unconditional: a chunk past the row's end reads its last one and counts as zeros.)
  constexpr int kAhead = 16;
  typedef typename std::conditional<BF16, uint2, uint4>::type Raw;  // four values
  Raw vr[kAhead];
  const int c0 = threadIdx.x * 4;
  auto load_v = [&](int k0, int c) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const uint32_t pick = sh.pick_id[k0 + k < K ? k0 + k : K - 1];
      vr[k] = *(const Raw*)((const char*)p.v + ((int64_t)pick * p.d + (c < p.d ? c : 0)) * kSize);
    }
  };
  {
    const uint4* const x = (const uint4*)((const char*)p.x + (int64_t)t * p.d * kSize);
    const int chunks = p.d / E;
    uint4 xr[4], ur[2][4];
    auto load_u = [&](int k, int q) {
#pragma unroll
      for (int i = 0; i < 4; ++i) xr[i] = x[q + 64 * i < chunks ? q + 64 * i : chunks - 1];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const uint32_t pick = (uint32_t)readlane_i32((int)eid, k + n * kWaves < K ? k + n * kWaves : k);
        const uint4* const u = (const uint4*)((const char*)p.u + (int64_t)pick * p.d * kSize);
#pragma unroll
        for (int i = 0; i < 4; ++i) ur[n][i] = u[q + 64 * i < chunks ? q + 64 * i : chunks - 1];
      }
    };
    if (w < K) load_u(w, l);
    load_v(0, c0);
    // Gates, on every wave, while the rows are under way: lane k has pick k's.
    const double s0 = f64_from_ord(sh.pick_score[0]);
    const float e = l < K ? expf((float)(f64_from_ord(sh.pick_score[l < K ? l : 0]) - s0)) : 0.0f;
    const float gate = e / wave_sum_uniform(e);
    if (w == 0 && l < K) {
      if (p.idx) p.idx[(int64_t)row * K + l] = (int32_t)eid;
      if (p.gates) p.gates[(int64_t)row * K + l] = gate;
    }
    for (int k = w; k < K; k += 2 * kWaves) {
      float acc[2] = {0.0f, 0.0f};
      for (int q = 0; q < chunks; q += 256) {
        if (k != w || q) load_u(k, q + l);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          // (both zeros: an infinity of u times a zero would not be one)
          const bool past = q + l + 64 * i >= chunks;
          if (past) xr[i] = make_uint4(0, 0, 0, 0);
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            if (past) ur[n][i] = make_uint4(0, 0, 0, 0);
            acc[n] = chunk_dot<BF16>(ur[n][i], xr[i], acc[n]);
          }
        }
      }
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const float h = wave_sum_uniform(acc[n]);
        if (l == k + n * kWaves && l < K) sh.a[l] = gate * activation(p.act_kind, h);
      }
    }
  }
  __syncthreads();
  float* const out = p.part + (int64_t)row * p.d;
  for (int c = c0; c < p.d; c += kThreads * 4) {
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k0 = 0; k0 < K; k0 += kAhead) {
      if (c != c0 || k0) load_v(k0, c);
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (k0 + k < K) {
          const float a = sh.a[k0 + k];
          float4 r;
          if constexpr (BF16) r = make_float4(bf16_lo(vr[k].x), bf16_hi(vr[k].x), bf16_lo(vr[k].y), bf16_hi(vr[k].y));
          else r = __builtin_bit_cast(float4, vr[k]);
          s.x = fmaf(a, r.x, s.x);
          s.y = fmaf(a, r.y, s.y);
          s.z = fmaf(a, r.z, s.z);
          s.w = fmaf(a, r.w, s.w);
        }
    }
    store_agent(out + c, s.x, s.y);
    store_agent(out + c + 2, s.z, s.w);
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0): this wave's stores are past L2
  __syncthreads();
  if (w == 0) list_finished(p, sh, l < p.ranges, t, l);
  __syncthreads();
  add_finished(p, sh, t, 0);
}

size_t up(size_t v) { return (v + 255) & ~(size_t)255; }
int pad(int n) { return (n + 3) / 4 * 4; }

}  // namespace

bool few_fits(const Shape& s) { return s.T <= kTokens && s.K <= kCandK; }

size_t few_ws_bytes(const Shape& s, int F) {
  return up((size_t)s.rows * (pad(s.nr) + pad(s.nc)) * 4) + up((size_t)kTokens * F * (s.bf16 ? 2 * kSplit : 4)) +
         up((size_t)s.rows * s.d * 4) + up(F ? (size_t)s.T * ((s.d + 15) / 16 * 16) * 4 : 0) + kCounts * 4;
}

hipError_t launch_few(const Shape& s, int F, const void* x, const void* keys_row, const void* keys_col, const void* u,
                      const void* v, const void* w_gu, const void* w_down, float* y, int32_t* idx, float* gates,
                      void* ws, hipStream_t st) {
  FewArgs p;
  p.x = x;
  p.keys[0] = keys_row;
  p.keys[1] = keys_col;
  p.u = u;
  p.v = v;
  p.w_gu = w_gu;
  p.w_down = w_down;
  p.y = y;
  p.idx = idx;
  p.gates = gates;
  p.T = (int)s.T;
  p.d = s.d;
  p.F = F;
  p.H = s.H;
  p.K = s.K;
  p.act_kind = s.act;
  p.dk = s.dk;
  p.col0 = s.col0;
  p.n[0] = s.nr;
  p.n[1] = s.nc;
  for (int i = 0; i < 2; ++i) {
    p.npad[i] = pad(p.n[i]);
    p.key_groups[i] = (int)(((int64_t)s.H * p.n[i] + 15) / 16);
  }
  p.down_groups = F ? (s.d + 15) / 16 : 0;
  p.ranges = F ? (p.down_groups + kRangeGroups - 1) / kRangeGroups : 1;
  p.span = F ? 16 * kRangeGroups : s.d;
  char* w = (char*)ws;
  p.count = (int*)w;
  w += kCounts * 4;
  p.logits = (float*)w;
  w += up((size_t)s.rows * (p.npad[0] + p.npad[1]) * 4);
  p.act = w;
  w += up((size_t)kTokens * F * (s.bf16 ? 2 * kSplit : 4));
  p.part = (float*)w;
  w += up((size_t)s.rows * s.d * 4);
  p.shared = (float*)w;
  const dim3 products((unsigned)(p.key_groups[0] + p.key_groups[1] + (F + 7) / 8));
  if (s.bf16) hipLaunchKernelGGL(few_products<true>, products, dim3(256), 0, st, p);
  else hipLaunchKernelGGL(few_products<false>, products, dim3(256), 0, st, p);
  const dim3 finish((unsigned)(s.rows + p.down_groups));
  const int n = s.nr > s.nc ? s.nr : s.nc;
#define OMNIMOE_FEW(R_)                                                                         \
  do {                                                                                          \
    if (s.bf16) hipLaunchKernelGGL((few_finish<true, R_>), finish, dim3(kThreads), 0, st, p);   \
    else hipLaunchKernelGGL((few_finish<false, R_>), finish, dim3(kThreads), 0, st, p);         \
  } while (0)
  if (n <= 256) OMNIMOE_FEW(4);
  else if (n <= 512) OMNIMOE_FEW(8);
  else if (n <= 1024) OMNIMOE_FEW(16);
  else if (n <= 2048) OMNIMOE_FEW(32);
  else OMNIMOE_FEW(64);
#undef OMNIMOE_FEW
  return hipGetLastError();
}

}  // namespace omnimoe
