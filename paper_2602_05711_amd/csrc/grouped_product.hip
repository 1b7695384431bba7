// Products of rows grouped by expert: position p of expert e has y_p = W_e x_p (or silu(G_e x_p) (U_e x_p), W_e being G_e's
// rows and then U_e's), dx_p = W_e^T dy_p and dW_e = sum over e's positions of dy_p x_p^T.
//
// Many rows an expert: tile products (tile_gemm.hpp, tile_spread.hpp) whose rows are gathered by position, task or token while
// they are copied to LDS. The experts' positions are cut into units of a tile's rows; a workgroup finds its unit from the
// offsets itself, so that the grid depends on the sizes alone: units past the last leave at once. Bound by the matrix cores
// beside the copies and by the tiles' starts and ends (8 to 14 us of a 256 x 256 tile's 60, 2048 summed values): 131072 rows
// of 2048 on 64 experts of 2048 x 2048 with SwiGLU 1020 to 1040 us, 1.07 PFLOP/s, 65536 rows' dx 590 and dW 665 us, 0.93 and
// 0.83 (calls back to back); the library's dense product of 131072 x 2048 x 2048 reaches 1.36. Without its copies the loop runs at 1.34 to 1.54. Two groups
// of waves that take turns at the products, and workgroups that go from tile to tile, were no faster (1065 and 1074 us).
// Few rows: the time is that of reading the weights of the experts that have rows, and of little beside it
// (few_tile.hpp): a unit is up to sixteen rows, a workgroup takes 16 or 32 weight rows and splits the summed index over its
// waves. 128 rows on 64 experts of 2048 x 2048: 87 to 90 us, 5.3 TB/s.
// Sums are fp32, rounded once; every result has one order of summation, so that it is the same on every run.
#include "few_tile.hpp"
#include "grouped_rows.hpp"
#include "internal.hpp"
#include "tile_gemm.hpp"
#include "tile_spread.hpp"
#include "vec8.hpp"

#include <math.h>

namespace omnimoe {
namespace {

// Rows gathered over a whole tensor, the summed index contiguous: an address a copy, since the tensor may be larger than
// 32-bit offsets reach.
template <class T, int R, int NW>
struct RowOperand : TileOperand<T, R, false, NW> {
  typedef TileOperand<T, R, false, NW> Tile;
  const char* ptr[Tile::kCopies];

  template <class Row>
  __device__ __forceinline__ void init(const void* p, int64_t ld, int wid, int lane, Row row) {
    this->lds = wid * Tile::kCopies * 1024;
#pragma unroll
    for (int i = 0; i < Tile::kCopies; ++i) {
      const int at = (wid * Tile::kCopies + i) * 64 + lane, lrow = at / 8;
      ptr[i] = (const char*)p + ((int64_t)row(lrow) * ld + Tile::place(lrow, at % 8) * Tile::kPer) * T::kSize;
    }
  }
  __device__ __forceinline__ void copy(unsigned char* st, int at, int kt, int K, int wid, int lane) const {
    const int64_t skip = (int64_t)kt * T::kStep * T::kSize;
    const int left = K - kt * T::kStep;
#pragma unroll
    for (int i = 0; i < Tile::kCopies; ++i) {
      const char* p = ptr[i] + skip;
      p = Tile::chunk_k(i, lane, wid) < left ? p : (const char*)&tile_zeros;
      __builtin_amdgcn_global_load_lds((const void*)p, (tg_lds_ptr)(st + (at + this->lds + i * 1024)), 16, 0, 0);
    }
  }
  __device__ __forceinline__ void copy(unsigned char* st, int at, int64_t, int kt, int K, int wid, int lane) const {
    copy(st, at, kt, K, wid, lane);
  }
};

// The rows that the stages' positions name, by x's order and by dy's, in LDS: rows[kt % 4] from before stage kt's copies on.
// Wave 0 brings them, a position a lane: an entry of perm is loaded a stage before it is looked at, when nothing has to be
// waited for (loads return in order, behind the copies issued before them).
struct SumRows {
  RowOrder x, dy;
  int first, count;
  int2 (*rows)[64];
  int next;  // (the lane's entry that was loaded last)

  __device__ __forceinline__ int entry(int k) const { return x.perm ? x.perm[first + (k < count ? k : count - 1)] : 0; }
  __device__ __forceinline__ void fetch(int k) { next = entry(k); }
  __device__ __forceinline__ void put(int kt, int k) {
    const int p = first + k, t = x.perm ? next : p;
    rows[kt & 3][lane_id()] = k < count ? make_int2(x.of(p, t), dy.of(p, t)) : make_int2(-1, -1);
  }
  // The first N stages' rows, and the next one's entries of perm, all loaded together.
  template <int STEP, int N>
  __device__ __forceinline__ void begin() {
    int t[N + 1];
#pragma unroll
    for (int kt = 0; kt <= N; ++kt) t[kt] = entry(kt * STEP + lane_id());
#pragma unroll
    for (int kt = 0; kt < N; ++kt) {
      next = t[kt];
      put(kt, kt * STEP + lane_id());
    }
    next = t[N];
  }
};

// Rows as the summed index: stage kt holds positions first + kt kStep .. of `count`, R of their columns. BRINGS: its copies
// bring the next stage's rows.
template <class T, int R, int NW, bool DY, bool BRINGS>
struct SumOperand : TileOperand<T, R, true, NW> {
  typedef TileOperand<T, R, true, NW> Tile;
  static_assert(T::kStep <= 64, "a wave's lanes");
  const char* from[Tile::kCopies];
  int ld;
  SumRows* rows;

  __device__ __forceinline__ void init(const void* p, int width, int c0, SumRows* rows_, int wid, int lane) {
    ld = width * T::kSize, rows = rows_;
    this->lds = wid * Tile::kCopies * 1024;
#pragma unroll
    for (int i = 0; i < Tile::kCopies; ++i) {
      const int at = (wid * Tile::kCopies + i) * 64 + lane, lrow = at / Tile::kRowChunks;
      const int c = c0 + Tile::place(lrow, at % Tile::kRowChunks) * Tile::kPer;
      from[i] = (const char*)p + (int64_t)(c < width ? c : width - Tile::kPer) * T::kSize;
    }
  }
  __device__ __forceinline__ void copy(unsigned char* st, int at, int kt, int K, int wid, int lane) const {
#pragma unroll
    for (int i = 0; i < Tile::kCopies; ++i) {
      const int2 both = rows->rows[kt & 3][((wid * Tile::kCopies + i) * 64 + lane) / Tile::kRowChunks];
      const int row = DY ? both.y : both.x;
      const char* p = from[i] + (int64_t)row * ld;
      p = row >= 0 && K > 0 ? p : (const char*)&tile_zeros;
      __builtin_amdgcn_global_load_lds((const void*)p, (tg_lds_ptr)(st + (at + this->lds + i * 1024)), 16, 0, 0);
    }
  }
  __device__ __forceinline__ void copy(unsigned char* st, int at, int64_t, int kt, int K, int wid, int lane) const {
    copy(st, at, kt, K, wid, lane);
    if constexpr (BRINGS)
      if (wid == 0 && (kt + 1) * T::kStep < K) {
        rows->put(kt + 1, (kt + 1) * T::kStep + lane);
        rows->fetch((kt + 2) * T::kStep + lane);
      }
  }
};

struct GroupedArgs {
  const void *in, *w;
  void* out;
  const int32_t* offsets;
  int N, M, k, n;  // k: the summed width, n: the result's
  RowOrder in_rows, out_rows;
  unsigned block0;
};

// A wave's 32 x 32 block of results, of which this lane has sixteen values of b's row lane % 32 in fours (a's rows 8 q + 4 (lane /
// 32) + e), to the memory of that row; there(c): whether columns c .. c + 7 (fp32: c + 3) exist and are wanted. Rounded to
// bf16, fours change places between the lanes (v_permlane32_swap) so that a store is 16 bytes a lane, 32 a row instead of 16:
// gate and up projection of 131072 rows 1064 -> 1001 us. (64 a row, with v_permlane16_swap: 1018.)
template <class T, class There>
__device__ __forceinline__ void put_block(const float (&v)[16], int lane, void* to, There there) {
  if constexpr (T::kSize == 2) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const auto x = __builtin_amdgcn_permlane32_swap(bf16_pair(v[8 * h + 2 * e], v[8 * h + 2 * e + 1]),
                                                        bf16_pair(v[8 * h + 4 + 2 * e], v[8 * h + 5 + 2 * e]), false, false);
        w[e] = x[0], w[2 + e] = x[1];
      }
      const int c = 16 * h + 8 * (lane >> 5);
      if (there(c)) *(uint4*)((uint16_t*)to + c) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  } else {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int c = 8 * q + 4 * (lane >> 5);
      if (there(c)) *(float4*)((float*)to + c) = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
    }
  }
}

// TM positions x TN weight rows (SWIGLU: TN / 2 gate rows and the same features' up rows, in blocks of 32 in turn, so that a
// wave holds both) a workgroup of WR x WC waves. TRANSPOSED: the summed index is the weights' row (dx).
template <class T, int TM, int TN, int WR, int WC, bool TRANSPOSED, bool SWIGLU>
__global__ __launch_bounds__(64 * WR * WC) void grouped_tile_kernel(GroupedArgs p) {
  constexpr int NW = WR * WC, MJ = TM / WR / 32, NI = TN / WC / 32, FN = SWIGLU ? TN / 2 : TN;
  constexpr bool kSpread = TM == 256 && SWIGLU, kRing = TM < 256;
  static_assert(!SWIGLU || (NI % 2 == 0 && !TRANSPOSED), "a wave's gate and up rows");
  typedef typename T::elem elem;
  __shared__ __attribute__((aligned(1024))) unsigned char st0[(TM + TN) * 128], st1[(TM + TN) * 128];
  __shared__ __attribute__((aligned(1024))) unsigned char st2[kRing ? (TM + TN) * 128 : 16], st3[kRing ? (TM + TN) * 128 : 16];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wid / WC, wc = wid % WC;
  const int tiles_n = (p.n + FN - 1) / FN;
  // neighbouring tiles, which share rows or weights, go to one XCD
  RowUnit u;
  int tile = -1;
  find_unit<64 * NW>(p.offsets, p.N, p.M, TM, (int*)st0, [&](int total) {
    const int64_t all = (int64_t)total * tiles_n;
    const unsigned block = p.block0 + blockIdx.x;
    if (block >= all) return -1;
    const unsigned item = (unsigned)xcd_contiguous(block, all), unit = item / (unsigned)tiles_n;
    tile = __builtin_amdgcn_readfirstlane((int)(item - unit * tiles_n));
    return (int)unit;
  }, u);
  if (tile < 0) return;
  __syncthreads();
  const int n0 = tile * FN;
  int a0[NI], b0[MJ];
#pragma unroll
  for (int i = 0; i < NI; ++i) a0[i] = (wc * NI + i) * 32;
#pragma unroll
  for (int j = 0; j < MJ; ++j) b0[j] = (wr * MJ + j) * 32;
  tg_f32x16 acc[NI][MJ];
  tile_zero(acc);
  RowOperand<T, TM, NW> b;
  b.init(p.in, p.k, wid, lane, [&](int r) {
    const int row = p.in_rows(u.first + (r < u.count ? r : u.count - 1));
    return row < 0 ? 0 : row;
  });
  typename std::conditional<kSpread || kRing, SpreadOperand<T, TN, TRANSPOSED, NW>, TileOperand<T, TN, TRANSPOSED, NW>>::type a;
  const elem* const w = (const elem*)p.w + (int64_t)u.expert * (SWIGLU ? 2 : 1) * p.n * p.k;
  if constexpr (TRANSPOSED)
    a.init(w, p.n, wid, lane, [&](int r) { return n0 + r < p.n ? n0 + r : p.n - a.kPer; });
  else
    a.init(w, p.k, wid, lane, [&](int r) {
      const int f = n0 + (SWIGLU ? (r >> 6) * 32 + (r & 31) : r), c = f < p.n ? f : p.n - 1;
      return SWIGLU && (r & 32) ? p.n + c : c;
    });
  if constexpr (kSpread) {
    spread_sum<T>(a, b, p.k, a0, b0, wr * (TM / WR) < u.count, st0, st1, wid, lane, acc, [](int) {});
  } else if constexpr (kRing) {
    ring_sum<T>(a, b, p.k, a0, b0, st0, st1, st2, st3, wid, lane, acc);
  } else {
    const TileRange all[2] = {{p.k, 0, 0}, {0, 0, 0}};
    tile_sum<T>(a, b, all, a0, b0, st0, st1, wid, lane, acc);
  }
  int out[MJ];  // (looked up together: a wait for each would be a fifth of the stores' time)
#pragma unroll
  for (int j = 0; j < MJ; ++j) {
    const int r = b0[j] + (lane & 31);
    out[j] = p.out_rows.task(u.first + (r < u.count ? r : u.count - 1));
  }
#pragma unroll
  for (int j = 0; j < MJ; ++j) {
    const int r = b0[j] + (lane & 31), row = r < u.count ? p.out_rows.of(u.first + r, out[j]) : -1;
#pragma unroll
    for (int i = 0; i < NI; i += SWIGLU ? 2 : 1) {
      float v[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] = acc[i][j][e];
      if constexpr (SWIGLU) {
        constexpr bool kBf16 = T::kSize == 2;
        // (the bits of negative values, as whole numbers, are in the order of their magnitude and above all positive ones)
        uint32_t low = 0;
#pragma unroll
        for (int e = 0; e < 16; ++e) low = max(low, __float_as_uint(v[e]));
        if (__any(low > __float_as_uint(kDeepGate))) {  // a gate of the block's is below kDeepGate
#pragma unroll
          for (int e = 0; e < 16; ++e) v[e] = swiglu<kBf16>(v[e], acc[i + 1][j][e]);
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) v[e] = swiglu_near<kBf16>(v[e], acc[i + 1][j][e]);
        }
      }
      const int f = n0 + (SWIGLU ? a0[i] / 2 : a0[i]);
      put_block<T>(v, lane, (elem*)p.out + (int64_t)row * p.n + f, [&](int c) { return row >= 0 && f + c < p.n; });
    }
  }
}

// 16 RB weight rows (SWIGLU: half of them gate rows, in turn) for a unit of up to sixteen positions.
template <bool BF16, int RB, bool SWIGLU, int W>
__global__ __launch_bounds__(64 * W) void grouped_few_kernel(GroupedArgs p, int groups) {
  constexpr int E = Chunk<BF16>::kElems, kSize = BF16 ? 2 : 4, FB = SWIGLU ? RB / 2 : RB;
  typedef typename std::conditional<BF16, uint16_t, float>::type elem;
  __shared__ f32x4 tiles[W][RB][64];
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned block = p.block0 + blockIdx.x;
  const int want = block / (unsigned)groups, f0 = (int)(block % (unsigned)groups) * 16 * FB;
  RowUnit u;
  if (find_unit<64 * W>(p.offsets, p.N, p.M, 16, (int*)tiles, [&](int) { return want; }, u) <= want) return;
  __syncthreads();
  const int pos = u.first + ((l & 15) < u.count ? (l & 15) : u.count - 1), task = p.in_rows.task(pos);
  const int at = p.in_rows.of(pos, task);
  const uint4* const tok[1] = {(const uint4*)((const char*)p.in + (int64_t)(at < 0 ? 0 : at) * p.k * kSize)};
  const uint4* row[RB];
  const char* const weights = (const char*)p.w + (int64_t)u.expert * (SWIGLU ? 2 : 1) * p.n * p.k * kSize;
#pragma unroll
  for (int b = 0; b < RB; ++b) {
    const int f = f0 + 16 * (SWIGLU ? b / 2 : b) + (l & 15), c = f < p.n ? f : p.n - 1;
    row[b] = (const uint4*)(weights + (int64_t)(SWIGLU && (b & 1) ? p.n + c : c) * p.k * kSize);
  }
  f32x4 acc[RB];
  wave_tile<BF16, RB, 1, 1, W>(row, tok, p.k / E, w, acc);
  add_tiles(acc, tiles, w, l);
  if (w || (l & 15) >= u.count) return;
  const int to = p.out_rows.of(pos, task);
  if (to < 0) return;
  elem* const out = (elem*)p.out + (int64_t)to * p.n;
#pragma unroll
  for (int b = 0; b < RB; b += SWIGLU ? 2 : 1) {
    const int f = f0 + 16 * (SWIGLU ? b / 2 : b) + 4 * (l >> 4);
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

struct GroupedSumArgs {
  const void *x, *dy;
  void* dw;
  float* part;  // [parts][N][n][k]
  const int32_t* offsets;
  int N, M, n, k;
  RowOrder x_rows, y_rows;
  int parts;
  unsigned block0, blocks;
};

// Experts' rows may be very uneven. 16 to 64 of them, a multiple of eight, go to the XCDs by their rank in rows, to and fro
// (the first eight to XCDs 0 to 7, the next to 7 to 0, ...), so that each has about as many rows, the longest first; all of
// an expert's tiles stay on one XCD, whose L2 they share. Fewer experts' tiles go over all XCDs, the longest expert's first
// (eight experts of 2048 x 2048, 16384 rows, both gradients with tiles of 128: 344 us, with an XCD each 413). Other numbers of
// experts go in their own order, in which the XCD of the longest ones may end last. Returns the expert of rank `want`.
__device__ __forceinline__ int expert_of_rank(const int32_t* offsets, int N, int M, int want) {
  const int l = lane_id(), e = l < N ? l : N - 1;
  const int lo = expert_start(offsets, e, M), hi = expert_start(offsets, e + 1, M), rows = l < N ? (hi > lo ? hi - lo : 0) : -1;
  int rank = 0;
  for (int i = 0; i < N; ++i) {
    const int other = __builtin_amdgcn_readlane(rows, i);
    rank += other > rows || (other == rows && i < l);
  }
  return __builtin_ctzll(__ballot(rank == want));
}

// A tile of dW_e: TM of y's columns x TN of x's, one part of e's positions. 65536 rows on 64 experts of 2048 x 2048, some with
// three times others' rows: 665 us (with every copy looking up its row by itself 1560, experts in their own order 846).
template <class T, int TM, int TN, int WR, int WC>
__global__ __launch_bounds__(64 * WR * WC) void grouped_sum_kernel(GroupedSumArgs p) {
  constexpr int NW = WR * WC, MJ = TM / WR / 32, NI = TN / WC / 32;
  typedef typename T::elem elem;
  __shared__ __attribute__((aligned(1024))) unsigned char st0[(TM + TN) * 128], st1[(TM + TN) * 128];
  __shared__ int2 slots[4][64];
  const int lane = threadIdx.x & 63, wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wr = wid / WC, wc = wid % WC;
  const unsigned tiles_k = (p.k + TN - 1) / TN, tiles_n = (p.n + TM - 1) / TM, each = tiles_k * tiles_n * p.parts;
  const unsigned block = p.block0 + blockIdx.x;
  unsigned item;
  int e;
  if (p.offsets && p.N > 1 && p.N < 16) {
    const unsigned rank = block / each;
    item = block - rank * each;
    e = __builtin_amdgcn_readfirstlane(expert_of_rank(p.offsets, p.N, p.M, (int)rank));
  } else if (p.offsets && p.N <= 64 && p.N % 8 == 0) {
    const unsigned xcd = block % 8, at = block / 8, turn = at / each;
    item = at - turn * each;
    e = __builtin_amdgcn_readfirstlane(expert_of_rank(p.offsets, p.N, p.M, (int)(8 * turn + (turn & 1 ? 7 - xcd : xcd))));
  } else {
    const unsigned at = (unsigned)xcd_contiguous(block, p.blocks);
    e = (int)(at / each);
    item = at - e * each;
  }
  const unsigned part_ = item / (tiles_k * tiles_n), tile = item - part_ * tiles_k * tiles_n;
  const int part = (int)part_, tn = (int)(tile / tiles_k), tk = (int)(tile - tn * tiles_k);
  const int lo = expert_start(p.offsets, e, p.M), hi = expert_start(p.offsets, e + 1, p.M);
  const int all_rows = hi > lo ? hi - lo : 0, per = ((all_rows + p.parts - 1) / p.parts + 63) / 64 * 64;
  const int64_t skip = (int64_t)part * per;
  const int first = (int)(lo + skip), count = skip >= all_rows ? 0 : all_rows - skip < per ? (int)(all_rows - skip) : per;
  int a0[NI], b0[MJ];
#pragma unroll
  for (int j = 0; j < MJ; ++j) b0[j] = (wr * MJ + j) * 32;
#pragma unroll
  for (int i = 0; i < NI; ++i) a0[i] = (wc * NI + i) * 32;
  tg_f32x16 acc[NI][MJ];
  tile_zero(acc);
  SumRows rows{p.x_rows, p.y_rows, first, count, slots, 0};
  SumOperand<T, TN, NW, false, false> a;
  SumOperand<T, TM, NW, true, true> b;
  a.init(p.x, p.k, (int)tk * TN, &rows, wid, lane);
  b.init(p.dy, p.n, (int)tn * TM, &rows, wid, lane);
  if (count) {
    if (wid == 0) rows.begin<T::kStep, TM == 256 ? 3 : 1>();
    __syncthreads();
  }
  if constexpr (TM == 256) {
    spread_sum<T>(a, b, count, a0, b0, true, st0, st1, wid, lane, acc, [&](int s) {
      if (wid) return;
      rows.put(s + 3, (s + 3) * T::kStep + lane);
      rows.fetch((s + 4) * T::kStep + lane);
    });
  } else {
    const TileRange all[2] = {{count, 0, 0}, {0, 0, 0}};
    tile_sum<T>(a, b, all, a0, b0, st0, st1, wid, lane, acc);
  }
#pragma unroll
  for (int j = 0; j < MJ; ++j) {
    const int n = tn * TM + b0[j] + (lane & 31);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      const int k = tk * TN + a0[i];
      const int64_t at = ((int64_t)e * p.n + n) * p.k + k;
      const auto there = [&](int c) { return n < p.n && k + c < p.k; };
      float v[16];
#pragma unroll
      for (int c = 0; c < 16; ++c) v[c] = acc[i][j][c];
      if (p.parts > 1) put_block<F32>(v, lane, p.part + (int64_t)part * p.N * p.n * p.k + at, there);
      else put_block<T>(v, lane, (elem*)p.dw + at, there);
    }
  }
}

template <class T>
__global__ __launch_bounds__(256) void grouped_add_kernel(const float* __restrict__ part, void* __restrict__ dw, int64_t size,
                                                          int parts) {
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < size; i += (int64_t)gridDim.x * 1024) {
    float4 v = *(const float4*)(part + i);
    for (int z = 1; z < parts; ++z) {
      const float4 s = *(const float4*)(part + z * size + i);
      v.x += s.x;
      v.y += s.y;
      v.z += s.z;
      v.w += s.w;
    }
    put4((typename T::elem*)dw + i, v.x, v.y, v.z, v.w);
  }
}

// Units of R rows that M positions of N experts can have at most.
int64_t most_units(int64_t M, int N, int R) {
  const int64_t n = M / R + N;
  return n < M ? n : M;
}
RowOrder rows(const Shape& s, const int32_t* perm, int order) { return RowOrder::make(perm, (int)s.M, order, s.hk); }
int64_t cut(int64_t v, int64_t by) { return (v + by - 1) / by; }

// What bf16 tiles take, in us: a stage of r workgroups that share a compute unit stage[r] (between whole r a straight line;
// stage[0]: of a few workgroups on the whole card), at most `most` of them, and a tile's start and end `ends`. `tiles`
// workgroups of `stages` stages run in whole rounds of 256 `most` and a rest.
struct TileTime {
  int most;
  double stage[5], ends;
};
constexpr TileTime kTime256 = {1, {1.25, 1.65}, 9}, kTime128 = {1, {0.5, 0.66}, 2.7}, kTime64 = {2, {0.24, 0.3, 0.55}, 2.2};
constexpr TileTime kTime64Swiglu = {1, {0.43, 0.47}, 2.3};
constexpr TileTime kSum256 = kTime256, kSum128 = {2, {0.6, 0.75, 1.1}, 5}, kSum64 = {4, {0.45, 0.45, 0.55, 0.75, 0.95}, 4};
// (grouped_sum_kernel's two stages and its rows' numbers, in a compute unit's 160 KiB of LDS)
constexpr int sum_most(int side) { return 160 * 1024 / (2 * 2 * side * 128 + 4 * 64 * (int)sizeof(int2)); }
static_assert(kSum256.most == sum_most(256) && kSum128.most == sum_most(128) && kSum64.most == sum_most(64), "LDS");
double tiles_time(const TileTime& t, double tiles, double stages) {
  const double slots = 256.0 * t.most, rounds = floor(tiles / slots), r = (tiles - rounds * slots) / 256.0;
  const double whole = rounds * (stages * t.stage[t.most] + t.ends);
  if (r <= 0) return whole;
  const int at = (int)r;
  return whole + stages * (t.stage[at] + (r - at) * (t.stage[at + 1] - t.stage[at])) + t.ends;
}

// The tile's side, by these times with half a unit more an expert than its rows fill. Rows, experts, width, of 2048 x 2048
// matrices (us for 64, 128, 256): 1024, 1: 19, 20, 51; 4096, 1: 76, 45, 53; 4096, 16: 93, 70, 64; 16384, 64: 352, 257, 228;
// 8192, 64, whose weights take 110 us to read: 207, 171, 193 (the rule takes 256); of 1024 x 1024: 16384, 16: 80, 65, 63.
// fp32: 64 (its products take eight times bf16's time, so that a tile's copies are nothing beside them: 8192 rows,
// 1024 x 1024, 16 experts 169 us, 102 TFLOP/s).
int tile_side(bool bf16, bool swiglu, int64_t M, int N, int k, int n) {
  if (!bf16) return 64;
  int best = 64;
  double least = 0;
  for (const int side : {64, 128, 256}) {
    const double some = (double)M / side + (N > 1 ? 0.5 * N : 0.0), units = some < (double)M ? some : (double)M;
    const TileTime& t = side == 256 ? kTime256 : side == 128 ? kTime128 : swiglu ? kTime64Swiglu : kTime64;
    const double us = tiles_time(t, ceil(units) * cut(n, side == 64 && swiglu ? 128 : side), cut(k, 64));
    if (side == 64 || us < least) best = side, least = us;
  }
  return best;
}

template <class T, bool TRANSPOSED, bool SWIGLU>
hipError_t tiles(const GroupedArgs& p, hipStream_t st) {
  const int width = SWIGLU ? 2 * p.n : p.n;
  auto go = [&](auto kernel, int tm, int tn, int threads) -> hipError_t {
    return launch_numbered(kernel, most_units(p.M, p.N, tm) * cut(p.n, SWIGLU ? tn / 2 : tn), threads, st, p);
  };
  const int side = tile_side(T::kSize == 2, SWIGLU, p.M, p.N, p.k, width);
  if constexpr (T::kSize == 2) {
    if (side == 256) return go(grouped_tile_kernel<T, 256, 256, 2, 4, TRANSPOSED, SWIGLU>, 256, 256, 512);
    if (side == 128) return go(grouped_tile_kernel<T, 128, 128, 4, 2, TRANSPOSED, SWIGLU>, 128, 128, 512);
  }
  if constexpr (SWIGLU) return go(grouped_tile_kernel<T, 64, 128, 2, 2, TRANSPOSED, SWIGLU>, 64, 128, 256);
  else return go(grouped_tile_kernel<T, 64, 64, 2, 2, TRANSPOSED, SWIGLU>, 64, 64, 256);
}

template <bool BF16, bool SWIGLU, int RB, int W>
hipError_t few_launch(const GroupedArgs& p, int64_t units, hipStream_t st) {
  const int64_t groups = cut(p.n, SWIGLU ? 8 * RB : 16 * RB);
  return launch_numbered(grouped_few_kernel<BF16, RB, SWIGLU, W>, units * groups, 64 * W, st, p, (int)groups);
}
// Two row blocks a workgroup (SwiGLU: gate and up rows), one where two would leave compute units idle (a matrix of 2048 x 8192,
// one token, before tiles took it: 13.7 us instead of 19.3); eight waves where each has four steps of its loads in flight (64
// experts of 2048 x 2048, 4 and 64 tokens: 47 and 121 us, with four waves 54 and 126), else four (16 fp32 experts of 512 x 1024,
// 8 tokens: 8.4 us, with eight 10.1). Four row blocks: 62 and 144 us.
template <bool BF16, bool SWIGLU>
hipError_t few(const GroupedArgs& p, hipStream_t st) {
  const int64_t units = most_units(p.M, p.N, 16);
  if (p.k / Chunk<BF16>::kElems < 256) return few_launch<BF16, SWIGLU, 2, 4>(p, units, st);
  if constexpr (!SWIGLU) {
    if (units * cut(p.n, 16) < 512) return few_launch<BF16, SWIGLU, 1, 8>(p, units, st);
  }
  return few_launch<BF16, SWIGLU, 2, 8>(p, units, st);
}

// Whether a pass over the weights for every sixteen positions is faster than tiles of 64, whose copies bring the weights as
// fast once there is a workgroup for every other compute unit. us of both, bf16: 2048 x 2048, one expert, 64 positions 8.5 and
// 10.1, 96 13.8 and 10.3; 16 experts, 32 28 and 20; 64 experts, 8 14.9 and 11.7, 512 113 and 98; one of 2048 x 8192, 64 26 and
// 10.5. SwiGLU, whose tiles are one a compute unit, 2048 x 1024: one expert, 128 14.0 and 16.1; 16 experts, 128 37 and 31; 64
// experts, 128 78 and 81, 256 95 and 105. fp32, whose tiles' products take longer: 1024 x 1024, one expert, 192 15.8 and 21.6;
// 16 experts, 256 27 and 22; 64 experts, 512 75 and 79; 512 x 512, 16 experts, 256 9.0 and 12.4.
bool few_rows(bool bf16, bool swiglu, int64_t M, int N, int n) {
  if (!bf16) return M <= 192 || M <= 8 * (int64_t)N || M * n <= 1 << 17;
  const int64_t units = most_units(M, N, 16);
  if (swiglu) return units <= 8 || (N >= 32 && M <= 6 * (int64_t)N);
  return units <= 5 && most_units(M, N, 64) * cut(n, 64) < 128;
}

template <class T>
hipError_t forward(const GroupedArgs& p, bool swiglu, hipStream_t st) {
  if (few_rows(T::kSize == 2, swiglu, p.M, p.N, p.n)) return swiglu ? few<T::kSize == 2, true>(p, st) : few<T::kSize == 2, false>(p, st);
  return swiglu ? tiles<T, false, true>(p, st) : tiles<T, false, false>(p, st);
}

// The weight gradients' tiles, and parts of an expert's positions, of 512 at least, where the tiles leave compute units idle:
// by the same times, with a tile's sum more for the experts' unevenness, and parts' way through memory. Of 752 sizes (512 to
// 65536 rows, 1 to 256 experts of 512 x 264 to 4096 x 4096) the choice takes 1.02 times the fastest side's time in the mean. Rows,
// experts, matrices (us for 64, 128, 256): 16384, 8 of 2048 x 2048: 259, 174, 135; 32768, 16 of 1024 x 2048: 398, 257, 198;
// 16384, 1 of 2048 x 2048: 256, 166, 162; 16384, 16 of 1024 x 1024: 114, 76, 97; 8192, 12 of 512 x 512: 36, 45, 73.
struct SumPlan {
  int side, parts;
};
SumPlan sum_plan(const Shape& s, int k, int n) {
  SumPlan best{64, 1};
  double least = 0;
  for (const int side : {64, 128, 256}) {
    if (side > 64 && !s.bf16) break;
    const int64_t tiles = s.N * cut(k, side) * cut(n, side), wanted = 512 / tiles, most = s.M / s.N / 512;
    const int64_t cuts = wanted < most ? wanted : most;
    const int parts = cuts < 1 ? 1 : cuts > 32 ? 32 : (int)cuts;
    const TileTime& t = side == 256 ? kSum256 : side == 128 ? kSum128 : kSum64;
    const double stages = (double)s.M / s.N / parts / 64;
    const double us = tiles_time(t, (double)tiles * parts, stages) + stages * t.stage[1] +
                      (parts > 1 ? 3 + (2.0 * parts * 4 + 2) * s.N * k * n / 4e6 : 0.0);
    if (side == 64 || us < least) best = {side, parts}, least = us;
  }
  return best;
}

template <class T>
hipError_t sums(GroupedSumArgs p, int side, hipStream_t st) {
  auto go = [&](auto kernel, int threads) -> hipError_t {
    const int64_t grid = (int64_t)p.N * p.parts * cut(p.k, side) * cut(p.n, side);
    p.blocks = (unsigned)grid;
    return launch_numbered(kernel, grid, threads, st, p);
  };
  hipError_t e = hipSuccess;
  if constexpr (T::kSize == 2) {
    if (side == 256) e = go(grouped_sum_kernel<T, 256, 256, 2, 4>, 512);
    else if (side == 128) e = go(grouped_sum_kernel<T, 128, 128, 2, 4>, 512);
  }
  if (side == 64) e = go(grouped_sum_kernel<T, 64, 64, 2, 2>, 256);
  if (e || p.parts == 1) return e;
  const int64_t size = (int64_t)p.N * p.n * p.k, blocks = cut(size, 1024);
  hipLaunchKernelGGL(grouped_add_kernel<T>, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, st, p.part, p.dw,
                     size, p.parts);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_grouped_product(const Shape& s, const ProductShape& q, const void* x, const void* w,
                                  const int32_t* offsets, const int32_t* perm, void* y, hipStream_t st) {
  const GroupedArgs p{x, w, y, offsets, (int)s.N, (int)s.M, q.n_in, q.n_out, rows(s, perm, q.x_order), rows(s, perm, q.y_order), 0};
  return s.bf16 ? forward<BF16>(p, q.swiglu, st) : forward<F32>(p, q.swiglu, st);
}

hipError_t launch_grouped_dx(const Shape& s, const ProductShape& q, const void* dy, const void* w, const int32_t* offsets,
                             const int32_t* perm, void* dx, hipStream_t st) {
  const GroupedArgs p{dy, w, dx, offsets, (int)s.N, (int)s.M, q.n_out, q.n_in, rows(s, perm, q.y_order), rows(s, perm, q.x_order), 0};
  return s.bf16 ? tiles<BF16, true, false>(p, st) : tiles<F32, true, false>(p, st);
}

size_t grouped_dw_ws_bytes(const Shape& s, const ProductShape& q) {
  const int parts = sum_plan(s, q.n_in, q.n_out).parts;
  return parts > 1 ? (size_t)parts * s.N * q.n_in * q.n_out * 4 : 0;
}

hipError_t launch_grouped_dw(const Shape& s, const ProductShape& q, const void* x, const void* dy, const int32_t* offsets,
                             const int32_t* perm, void* dw, void* ws, hipStream_t st) {
  const SumPlan plan = sum_plan(s, q.n_in, q.n_out);
  const GroupedSumArgs p{x, dy, dw, (float*)ws, offsets, (int)s.N, (int)s.M, q.n_out, q.n_in, rows(s, perm, q.x_order),
                         rows(s, perm, q.y_order), plan.parts, 0, 0};
  return s.bf16 ? sums<BF16>(p, plan.side, st) : sums<F32>(p, plan.side, st);
}

}  // namespace omnimoe
