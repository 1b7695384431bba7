// The joint between a branch and the residual stream: for each token, with norm(v) = v / sqrt(mean(v^2) + eps),
//   x' = x + scale s b,  b = w_out norm(y),  s = sigmoid(gate);   n = w_in norm(x')
// and the way back. With rho = 1 / sqrt(mean(x'^2) + eps), r the same of y, xh = x' rho, yh = y r and u = w_in dn:
//   G  = dx' + rho (u - xh mean(u xh))                      dL/dx' and dL/dx
//   q  = G s scale w_out;  dy = r (q - yh mean(q yh))       (without w_out: yh = y and dy = q)
//   dgate = (1 - s) q yh, for one gate a token summed over the channels (the sum that dy needs)
//   dw_in = sum over the tokens of dn xh;  with S = sum of G s yh: dscale = w_out S, dw_out = scale S
// Both ways are bound by memory: every value is read and written once, a row lies in registers from its first read to its
// last use, and the way back forms the norms again instead of reading them. 16384 tokens, d = 2048, bf16: 64 us with a gate a
// token (5.2 TB/s), back 137 us and the columns' sums 5 with a gate a channel (139 together back to back, 4.8 TB/s; a large copy
// runs at 4.7); 4096 tokens, d = 8192, a gate a token: 75 and 117 us (4.5 TB/s). One token: 2.9 us, a launch's own time.
// Sums, norms and the joint itself are fp32; results are rounded to the layer's type once (n from the unrounded x').
#include "internal.hpp"
#include "vec8.hpp"

namespace omnimoe {
namespace {

struct JoinArgs {
  const void* x;  // back: x'
  const float* y;
  const void* gate;
  const float *w_out, *scale, *w_in;
  void *x_out, *n;
  const void *dx_out, *dn;
  void* dx;
  float* dy;
  void* dgate;
  float* part;  // [workgroups][2][d]: sums of G s yh, then of dn xh
  int64_t T;
  int d, gate_width;
  float eps;
};

// sigmoid(g) and what it leaves to 1, both to fp32's relative accuracy.
__device__ __forceinline__ float sigmoid(float g, float& rest) {
  const float e = expf(-fabsf(g)), b = 1.0f + e, r = __builtin_amdgcn_rcpf(b);
  const float big = fmaf(fmaf(-b, r, 1.0f), r, r), small = e * big;  // (1 <= b <= 2: a step of Newton's gives 1 / b)
  rest = g < 0.0f ? big : small;
  return g < 0.0f ? small : big;
}
__device__ __forceinline__ float sigmoid(float g) {
  float rest;
  return sigmoid(g, rest);
}

// Sums of N values over the workgroup's W waves, in wave order; every thread gets them. Two buffers in turn: a thread
// that writes one again has met every other at the barrier of the sums between.
template <int W, int N>
__device__ __forceinline__ void block_sums(float (&v)[N], float (&lds)[2][W][N], int& turn) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = wave_sum_uniform(v[i]);
  if constexpr (W > 1) {
    const int w = threadIdx.x >> 6;
    if (lane_id() == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) lds[turn][w][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = lds[turn][0][i];
#pragma unroll
      for (int k = 1; k < W; ++k) v[i] += lds[turn][k][i];
    }
    turn ^= 1;
  }
}

// Where the sum of a row's squares passes fp32's range they are formed of values times this: of at most 2^56, so that
// 2^15 squares sum to less than 2^128. (A value is multiplied with the norm's factor first, then with this, which rounds
// nothing that is not below fp32's normal values in the end.)
constexpr float kSmall = 0x1p-72f;
static_assert(kMaxWidth <= 1 << 15, "a row's squares");

__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u; }

__device__ __forceinline__ void load8f(const float* p, int64_t i, float (&v)[8]) { load8<false>(p, i, v); }

// One row a group of W waves, C chunks of eight values a lane: one wave up to d = 1024, whose sums need no barrier, then four,
// whose registers hold the row and the three vectors.
template <bool BF16, int W, int C>
__global__ __launch_bounds__(256) void join_kernel(JoinArgs p) {
  constexpr int kRows = 4 / W, NT = 64 * W;
  __shared__ float lds[2][W][1];
  int turn = 0;
  const int tid = W == 4 ? (int)threadIdx.x : lane_id(), q8 = p.d / 8;
  float a[C][8], w_in[C][8];
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const int at = c * NT + tid;
#pragma unroll
    for (int e = 0; e < 8; ++e) a[c][e] = w_in[c][e] = 1.0f;
    if (at >= q8) continue;
    if (p.w_in) load8f(p.w_in, at * 8, w_in[c]);
    if (p.y && p.scale) load8f(p.scale, at * 8, a[c]);
    if (p.y && p.w_out) {
      float w[8];
      load8f(p.w_out, at * 8, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) a[c][e] *= w[e];
    }
  }
  auto norm = [&](const float (&v)[C][8], float& pre, float& inv) {
    pre = 1.0f;
    for (;;) {
      float s[1] = {0.0f};
#pragma unroll
      for (int c = 0; c < C; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float z = v[c][e] * pre;
          s[0] = fmaf(z, z, s[0]);
        }
      block_sums<W>(s, lds, turn);
      s[0] = s[0] / (float)p.d + p.eps * pre * pre;
      inv = 1.0f / sqrtf(s[0]);
      if (finite(s[0]) || pre != 1.0f) return;
      pre = kSmall;
    }
  };
  for (int64_t t = (int64_t)blockIdx.x * kRows + (W == 4 ? 0 : threadIdx.x >> 6); t < p.T; t += (int64_t)gridDim.x * kRows) {
    float y[C][8], x[C][8], g[C][8];
    const float gate = p.y && p.gate_width == 1 ? (BF16 ? bf16_lo(((const uint16_t*)p.gate)[t]) : ((const float*)p.gate)[t]) : 0.0f;
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = c * NT + tid;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[c][e] = x[c][e] = g[c][e] = 0.0f;
      if (at >= q8) continue;
      load8<BF16>(p.x, t * p.d + at * 8, x[c]);
      if (p.y) {
        load8f(p.y, t * p.d + at * 8, y[c]);
        if (p.gate_width > 1) load8<BF16>(p.gate, t * p.d + at * 8, g[c]);
      }
    }
    float pre = 1.0f, inv = 1.0f;
    if (p.y) {
      if (p.w_out) norm(y, pre, inv);
      const float s = p.gate_width == 1 ? sigmoid(gate) : 1.0f;
#pragma unroll
      for (int c = 0; c < C; ++c) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float b = a[c][e] * (y[c][e] * inv * pre);
          b *= p.gate_width > 1 ? sigmoid(g[c][e]) : s;
          x[c][e] += b;
        }
        const int at = c * NT + tid;
        if (at < q8) store8<BF16>(p.x_out, t * p.d + at * 8, x[c]);
      }
    }
    if (!p.w_in) continue;
    norm(x, pre, inv);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int at = c * NT + tid;
      if (at >= q8) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[c][e] = w_in[c][e] * (x[c][e] * inv * pre);
      store8<BF16>(p.n, t * p.d + at * 8, x[c]);
    }
  }
}

// A row of the way back as it lies in memory, this thread's eight values of each.
template <bool BF16>
struct BackRow {
  Raw8<BF16> x, dn, dx_out, gate;
  Raw8<false> y;
  float token;
  __device__ __forceinline__ void zero() {
    x.zero(), dn.zero(), dx_out.zero(), gate.zero(), y.zero();
    token = 0.0f;
  }
  __device__ __forceinline__ void load(const JoinArgs& p, int64_t t, int c0, bool in) {
    if (p.y && p.gate_width == 1) token = BF16 ? bf16_lo(((const uint16_t*)p.gate)[t]) : ((const float*)p.gate)[t];
    if (!in) return;
    const int64_t at = t * p.d + c0;
    if (p.w_in) {
      x.load(p.x, at);
      dn.load(p.dn, at);
    }
    if (p.dx_out) dx_out.load(p.dx_out, at);
    if (p.y) y.load(p.y, at);
    if (p.y && p.gate_width > 1) gate.load(p.gate, at);
  }
};

// A row at a time a workgroup of W waves, eight values of each operand a thread; the next row's are on their way meanwhile
// (16384 tokens, d = 2048: 137 us; two rows at once with nothing on its way 191). A thread keeps its columns' sums over the
// rows. The vector units are busy for two fifths of the time, which is why a sigmoid's division is a reciprocal and one step.
template <bool BF16, int W>
__global__ __launch_bounds__(64 * W) void join_back_kernel(JoinArgs p) {
  __shared__ float lds3[2][W][3], lds1[2][W][1];
  int turn3 = 0, turn1 = 0;
  const int c0 = threadIdx.x * 8;
  const bool in = c0 < p.d;
  const float d1 = 1.0f / (float)p.d;
  const bool channel = p.y && p.gate_width > 1, token = p.y && p.gate_width == 1;
  BackRow<BF16> raw;
  raw.zero();
  const int64_t stride = gridDim.x;
  int64_t t = blockIdx.x;
  constexpr bool kAhead = W < 16;  // (sixteen waves' registers do not hold two rows)
  if (kAhead) raw.load(p, t, c0, in);
  float a[8], w_in[8], sum_s[8], sum_n[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) a[e] = 1.0f, w_in[e] = sum_s[e] = sum_n[e] = 0.0f;
  if (in) {
    if (p.w_in) load8f(p.w_in, c0, w_in);
    if (p.y && p.scale) load8f(p.scale, c0, a);
    if (p.y && p.w_out) {
      float w[8];
      load8f(p.w_out, c0, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) a[e] *= w[e];
    }
  }
  for (; t < p.T; t += stride) {
    float x[8], y[8], u[8], G[8], g[8], dn[8];
    if (!kAhead) {
      raw.zero();  // (whose registers are free between the rows, so that nothing is spilled)
      raw.load(p, t, c0, in);
    }
    raw.x.values(x);
    raw.dn.values(dn);
    raw.dx_out.values(G);
    raw.gate.values(g);
    raw.y.values(y);
    const float gate = raw.token;
    if (kAhead && t + stride < p.T) raw.load(p, t + stride, c0, in);
#pragma unroll
    for (int e = 0; e < 8; ++e) u[e] = w_in[e] * dn[e];
    // sums of x'^2, u x' and y^2
    float s3[3], pre_x = 1.0f, pre_y = 1.0f;
    for (bool again = false;;) {
      s3[0] = s3[1] = s3[2] = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float vx = x[e] * pre_x, vy = y[e] * pre_y;
        s3[0] = fmaf(vx, vx, s3[0]);
        s3[1] = fmaf(u[e], vx, s3[1]);
        s3[2] = fmaf(vy, vy, s3[2]);
      }
      block_sums<W>(s3, lds3, turn3);
      s3[0] = fmaf(s3[0], d1, p.eps * pre_x * pre_x), s3[2] = fmaf(s3[2], d1, p.eps * pre_y * pre_y);
      if (again || (finite(s3[0]) && finite(s3[2]))) break;  // (the sums are every thread's)
      if (!finite(s3[0])) pre_x = kSmall;
      if (!finite(s3[2])) pre_y = kSmall;
      again = true;
    }
    const float ix = 1.0f / sqrtf(s3[0]), m = s3[1] * ix * d1;
    const float iy = p.w_out ? 1.0f / sqrtf(s3[2]) : 1.0f;
    if (!p.w_out) pre_y = 1.0f;
    float rest = 0.0f;
    const float s = token ? sigmoid(gate, rest) : 1.0f;
    float sq[1] = {0.0f};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (p.w_in) {
        const float xh = x[e] * ix * pre_x;
        G[e] += ix * (u[e] - xh * m) * pre_x;
        sum_n[e] = fmaf(dn[e], xh, sum_n[e]);
      }
      y[e] = y[e] * iy * pre_y;  // yh
      const float Gs = G[e] * (channel ? sigmoid(g[e], g[e]) : s);
      sum_s[e] = fmaf(Gs, y[e], sum_s[e]);
      x[e] = Gs * a[e];  // q
      sq[0] = fmaf(x[e], y[e], sq[0]);
    }
    const int64_t at = t * p.d + c0;
    if (in) store8<BF16>(p.dx, at, G);
    if (!p.y) continue;
    if (channel && in) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = g[e] * (x[e] * y[e]);
      store8<BF16>(p.dgate, at, v);
    }
    if (!p.w_out) {  // dy = q, whatever y is
      if (in) store8<false>(p.dy, at, x);
      if (!token) continue;
    }
    block_sums<W>(sq, lds1, turn1);
    if (token && threadIdx.x == 0) {
      const float v = rest * sq[0];
      if constexpr (BF16) ((uint16_t*)p.dgate)[t] = bf16_rne(v);
      else ((float*)p.dgate)[t] = v;
    }
    if (!p.w_out || !in) continue;
    const float m2 = sq[0] * d1;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = iy * (x[e] - y[e] * m2) * pre_y;
    store8<false>(p.dy, at, y);
  }
  if (in) {
    float* const part = p.part + (int64_t)blockIdx.x * 2 * p.d + c0;
    store8<false>(part, 0, sum_s);
    store8<false>(part, p.d, sum_n);
  }
}

// The columns' sums of n workgroups, 32 columns a workgroup (3.9 and 5.0 us for 500 x 520 and 768 x 2048): 128 threads, four columns each, add every 128th one (eight of a
// thousand, in flight together), then 32 threads their sums in order.
constexpr int kColumnRows = 128;
__global__ __launch_bounds__(kColumnRows * 8) void join_columns_kernel(const float* __restrict__ part, int n, int d,
                                                                       const float* __restrict__ w_out,
                                                                       const float* __restrict__ scale, float* dw_out,
                                                                       float* dscale, float* dw_in) {
  __shared__ float lds[kColumnRows][33];
  __shared__ float four[4][32];
  const int col = threadIdx.x & 7, row = threadIdx.x >> 3, c = blockIdx.x * 32 + col * 4;
  const int which = blockIdx.y;  // 0: dw_out and dscale, 1: dw_in
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (c < d) {
    const float* const from = part + (int64_t)which * d + c;
#pragma unroll 8
    for (int i = row; i < n; i += kColumnRows) {
      const float4 s = *(const float4*)(from + (int64_t)i * 2 * d);
      v.x += s.x;
      v.y += s.y;
      v.z += s.z;
      v.w += s.w;
    }
  }
  lds[row][col * 4] = v.x;
  lds[row][col * 4 + 1] = v.y;
  lds[row][col * 4 + 2] = v.z;
  lds[row][col * 4 + 3] = v.w;
  __syncthreads();
  const int k = threadIdx.x & 31, quarter = threadIdx.x >> 5, c1 = blockIdx.x * 32 + k;
  float s = 0.0f;
  if (quarter < 4) {
#pragma unroll
    for (int i = 0; i < kColumnRows / 4; ++i) s += lds[quarter * (kColumnRows / 4) + i][k];
    four[quarter][k] = s;
  }
  __syncthreads();
  if (quarter || c1 >= d) return;
  s = (four[0][k] + four[1][k]) + (four[2][k] + four[3][k]);
  if (which) {
    if (dw_in) dw_in[c1] = s;
    return;
  }
  if (dscale) dscale[c1] = w_out ? w_out[c1] * s : s;
  if (dw_out) dw_out[c1] = scale ? scale[c1] * s : s;
}

int back_waves(int d) {
  int w = 1;
  while (w * 512 < d) w *= 2;
  return w;
}
// A workgroup's columns' sums cost a row's traffic; twelve waves a compute unit hide the rows' latency. 16384 tokens, d = 2048:
// 768 workgroups 139.6 us, 512 140.4, 256 147; 1000 tokens, 520, fp32: 500 12.4 us, 1000 13.9.
int back_groups(int64_t T, int d) {
  const int w = back_waves(d);
  const int64_t most = w > 8 ? 256 : 3072 / w, n = T <= 512 ? T : T <= 1024 ? 512 : T / 2;
  return (int)(n < most ? n : most);
}

static_assert(kMaxWidthF32 <= 4096 && kMaxWidth <= 8192, "the widest kernels");

template <bool BF16>
hipError_t join(const JoinArgs& p, hipStream_t st) {
  const int q8 = p.d / 8;
  auto go = [&](auto kernel, int rows) {
    const int64_t n = (p.T + rows - 1) / rows;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(n < 2048 ? n : 2048)), dim3(256), 0, st, p);
  };
  if (q8 <= 64) go(join_kernel<BF16, 1, 1>, 4);
  else if (q8 <= 128) go(join_kernel<BF16, 1, 2>, 4);
  else if (q8 <= 256) go(join_kernel<BF16, 4, 1>, 1);
  else if (q8 <= 512) go(join_kernel<BF16, 4, 2>, 1);
  if constexpr (BF16)
    if (q8 > 512) go(join_kernel<BF16, 4, 4>, 1);
  return hipGetLastError();
}

template <bool BF16>
hipError_t join_back(const JoinArgs& p, float* dw_out, float* dscale, float* dw_in, hipStream_t st) {
  const int n = back_groups(p.T, p.d), w = back_waves(p.d);
  if (n) {
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)n), dim3(64 * w), 0, st, p); };
    if (w == 1) go(join_back_kernel<BF16, 1>);
    else if (w == 2) go(join_back_kernel<BF16, 2>);
    else if (w == 4) go(join_back_kernel<BF16, 4>);
    else if (w == 8) go(join_back_kernel<BF16, 8>);
    if constexpr (BF16)
      if (w == 16) go(join_back_kernel<BF16, 16>);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  if (!dw_out && !dscale && !dw_in) return hipSuccess;
  hipLaunchKernelGGL(join_columns_kernel, dim3((unsigned)((p.d + 31) / 32), 2), dim3(kColumnRows * 8), 0, st, p.part, n, p.d, p.w_out,
                     p.scale, dw_out, dscale, dw_in);
  return hipGetLastError();
}

}  // namespace

size_t join_back_ws_bytes(int64_t T, int d) { return (size_t)back_groups(T, d) * 2 * d * 4; }

hipError_t launch_join(int64_t T, int d, bool bf16, float eps, int gate_width, const void* x, const float* y,
                       const void* gate, const float* w_out, const float* scale, const float* w_in, void* x_out, void* n,
                       hipStream_t st) {
  JoinArgs p{};
  p.x = x, p.y = y, p.gate = gate, p.w_out = w_out, p.scale = scale, p.w_in = w_in, p.x_out = x_out, p.n = n;
  p.T = T, p.d = d, p.gate_width = gate_width, p.eps = eps;
  return bf16 ? join<true>(p, st) : join<false>(p, st);
}

hipError_t launch_join_back(int64_t T, int d, bool bf16, float eps, int gate_width, const void* x_out, const float* y,
                            const void* gate, const float* w_out, const float* scale, const float* w_in,
                            const void* dx_out, const void* dn, void* dx, float* dy, void* dgate, float* dw_out,
                            float* dscale, float* dw_in, void* ws, hipStream_t st) {
  JoinArgs p{};
  p.x = x_out, p.y = y, p.gate = gate, p.w_out = w_out, p.scale = scale, p.w_in = w_in, p.dx_out = dx_out, p.dn = dn;
  p.dx = dx, p.dy = dy, p.dgate = dgate, p.part = (float*)ws;
  p.T = T, p.d = d, p.gate_width = gate_width, p.eps = eps;
  return bf16 ? join_back<true>(p, dw_out, dscale, dw_in, st) : join_back<false>(p, dw_out, dscale, dw_in, st);
}

}  // namespace omnimoe
