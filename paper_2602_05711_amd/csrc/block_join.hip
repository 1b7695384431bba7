// The joint between a branch and the residual stream: for each token, with norm(v) = v / sqrt(mean(v^2) + eps),
//   x' = x + scale s b,  b = w_out norm(y),  s = sigmoid(gate);   n = w_in norm(x')
// and the way back. With rho = 1 / sqrt(mean(x'^2) + eps), r the same of y, xh = x' rho, yh = y r and u = w_in dn:
//   G  = dx' + rho (u - xh mean(u xh))                      dL/dx' and dL/dx
//   q  = G s scale w_out;  dy = r (q - yh mean(q yh))       (without w_out: yh = y and dy = q)
//   dgate = (1 - s) q yh, for one gate a token summed over the channels (the sum that dy needs)
//   dw_in = sum over the tokens of dn xh;  with S = sum of G s yh: dscale = w_out S, dw_out = scale S
// Both ways are bound by memory: every value is read and written once, a row lies in registers from its first read to its
// last use, and the way back forms the norms again instead of reading them.
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
  const float e = expf(-fabsf(g)), big = 1.0f / (1.0f + e), small = e * big;
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

// Where a row's squares pass fp32's range they are formed of values times this.
constexpr float kSmall = 0x1p-70f;

__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7F800000u) != 0x7F800000u; }

__device__ __forceinline__ void load8f(const float* p, int64_t i, float (&v)[8]) { load8<false>(p, i, v); }

// One row a group of W waves, C chunks of eight values a lane.
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
      inv = 1.0f / sqrtf(s[0] / (float)p.d + p.eps * pre * pre);
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
          float b = a[c][e] * (y[c][e] * pre * inv);
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
      for (int e = 0; e < 8; ++e) x[c][e] = w_in[c][e] * (x[c][e] * pre * inv);
      store8<BF16>(p.n, t * p.d + at * 8, x[c]);
    }
  }
}

// R rows at a time a workgroup of W waves, eight values of each a thread. A thread keeps its columns' sums over the rows.
template <bool BF16, int W, int R>
__global__ __launch_bounds__(64 * W) void join_back_kernel(JoinArgs p) {
  __shared__ float lds3[2][W][3 * R], lds1[2][W][R];
  int turn3 = 0, turn1 = 0;
  const int c0 = threadIdx.x * 8;
  const bool in = c0 < p.d;
  const float d1 = 1.0f / (float)p.d;
  const bool channel = p.y && p.gate_width > 1, token = p.y && p.gate_width == 1;
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
  for (int64_t t0 = (int64_t)blockIdx.x * R; t0 < p.T; t0 += (int64_t)gridDim.x * R) {
    float x[R][8], y[R][8], dn[R][8], G[R][8], g[R][8];
#pragma unroll
    for (int i = 0; i < R; ++i) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[i][e] = y[i][e] = dn[i][e] = G[i][e] = g[i][e] = 0.0f;
      const int64_t t = t0 + i;
      if (t >= p.T) continue;
      if (token) g[i][0] = BF16 ? bf16_lo(((const uint16_t*)p.gate)[t]) : ((const float*)p.gate)[t];
      if (!in) continue;
      const int64_t at = t * p.d + c0;
      if (p.w_in) {
        load8<BF16>(p.x, at, x[i]);
        load8<BF16>(p.dn, at, dn[i]);
      }
      if (p.dx_out) load8<BF16>(p.dx_out, at, G[i]);
      if (p.y) load8f(p.y, at, y[i]);
      if (channel) load8<BF16>(p.gate, at, g[i]);
    }
    // sums of x'^2, u x' and y^2
    float s3[3 * R], pre_x[R], pre_y[R];
#pragma unroll
    for (int i = 0; i < R; ++i) pre_x[i] = pre_y[i] = 1.0f;
    for (bool again = false;;) {
      bool over = false;
#pragma unroll
      for (int i = 0; i < R; ++i) {
        float sx = 0.0f, su = 0.0f, sy = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float vx = x[i][e] * pre_x[i], vy = y[i][e] * pre_y[i];
          sx = fmaf(vx, vx, sx);
          su = fmaf(w_in[e] * dn[i][e], vx, su);
          sy = fmaf(vy, vy, sy);
        }
        s3[3 * i] = sx;
        s3[3 * i + 1] = su;
        s3[3 * i + 2] = sy;
      }
      block_sums<W>(s3, lds3, turn3);
#pragma unroll
      for (int i = 0; i < R; ++i) {
        if (!finite(s3[3 * i])) over = true, pre_x[i] = kSmall;
        if (!finite(s3[3 * i + 2])) over = true, pre_y[i] = kSmall;
      }
      if (!over || again) break;  // (the sums are every thread's)
      again = true;
    }
    float r[R], sq[R], s[R], rest[R];
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const float ix = 1.0f / sqrtf(s3[3 * i] * d1 + p.eps * pre_x[i] * pre_x[i]);
      const float iy = p.w_out ? 1.0f / sqrtf(s3[3 * i + 2] * d1 + p.eps * pre_y[i] * pre_y[i]) : 1.0f;
      const float m = s3[3 * i + 1] * ix * d1;
      if (!p.w_out) pre_y[i] = 1.0f;
      r[i] = iy;
      s[i] = token ? sigmoid(g[i][0], rest[i]) : 1.0f;
      sq[i] = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (p.w_in) {
          const float xh = x[i][e] * pre_x[i] * ix;
          G[i][e] += ix * (w_in[e] * dn[i][e] - xh * m) * pre_x[i];
          sum_n[e] = fmaf(dn[i][e], xh, sum_n[e]);
        }
        y[i][e] = y[i][e] * pre_y[i] * iy;  // yh
        const float Gs = G[i][e] * (channel ? sigmoid(g[i][e], g[i][e]) : s[i]);
        sum_s[e] = fmaf(Gs, y[i][e], sum_s[e]);
        x[i][e] = Gs * a[e];  // q
        sq[i] = fmaf(x[i][e], y[i][e], sq[i]);
      }
    }
    if (p.y) block_sums<W>(sq, lds1, turn1);
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const int64_t t = t0 + i;
      if (t >= p.T) break;
      if (token && threadIdx.x == 0) {
        const float v = rest[i] * sq[i];
        if constexpr (BF16) ((uint16_t*)p.dgate)[t] = bf16_rne(v);
        else ((float*)p.dgate)[t] = v;
      }
      if (!in) continue;
      const int64_t at = t * p.d + c0;
      store8<BF16>(p.dx, at, G[i]);
      if (!p.y) continue;
      const float m = p.w_out ? sq[i] * d1 : 0.0f;
      float v[8];
      if (channel) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = g[i][e] * (x[i][e] * y[i][e]);
        store8<BF16>(p.dgate, at, v);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = r[i] * (x[i][e] - y[i][e] * m) * pre_y[i];
      store8<false>(p.dy, at, v);
    }
  }
  if (in) {
    float* const part = p.part + (int64_t)blockIdx.x * 2 * p.d + c0;
    store8<false>(part, 0, sum_s);
    store8<false>(part, p.d, sum_n);
  }
}

// The columns' sums of n workgroups, sixteen columns a workgroup: sixteen threads a column add every sixteenth one, then the
// first of them those sums in order.
__global__ __launch_bounds__(256) void join_columns_kernel(const float* __restrict__ part, int n, int d,
                                                           const float* __restrict__ w_out,
                                                           const float* __restrict__ scale, float* dw_out, float* dscale,
                                                           float* dw_in) {
  __shared__ float lds[16][17];
  const int col = threadIdx.x & 15, row = threadIdx.x >> 4, c = blockIdx.x * 16 + col;
  const int which = blockIdx.y;  // 0: dw_out and dscale, 1: dw_in
  float v = 0.0f;
  if (c < d)
    for (int i = row; i < n; i += 16) v += part[((int64_t)i * 2 + which) * d + c];
  lds[row][col] = v;
  __syncthreads();
  if (row || c >= d) return;
#pragma unroll
  for (int i = 1; i < 16; ++i) v += lds[i][col];
  if (which) {
    if (dw_in) dw_in[c] = v;
    return;
  }
  if (dscale) dscale[c] = w_out ? w_out[c] * v : v;
  if (dw_out) dw_out[c] = scale ? scale[c] * v : v;
}

constexpr int kBackRows = 2;

int back_waves(int d) {
  int w = 1;
  while (w * 512 < d) w *= 2;
  return w;
}
int back_groups(int64_t T, int d) {
  const int w = back_waves(d);
  const int64_t n = (T + kBackRows - 1) / kBackRows, most = w > 8 ? 256 : 2048 / w;
  return (int)(n < most ? n : most);
}

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
  else go(join_kernel<BF16, 4, 4>, 1);
  return hipGetLastError();
}

template <bool BF16>
hipError_t join_back(const JoinArgs& p, float* dw_out, float* dscale, float* dw_in, hipStream_t st) {
  const int n = back_groups(p.T, p.d), w = back_waves(p.d);
  if (n) {
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)n), dim3(64 * w), 0, st, p); };
    if (w == 1) go(join_back_kernel<BF16, 1, kBackRows>);
    else if (w == 2) go(join_back_kernel<BF16, 2, kBackRows>);
    else if (w == 4) go(join_back_kernel<BF16, 4, kBackRows>);
    else if (w == 8) go(join_back_kernel<BF16, 8, kBackRows>);
    else go(join_back_kernel<BF16, 16, kBackRows>);
    if (const hipError_t e = hipGetLastError()) return e;
  }
  if (!dw_out && !dscale && !dw_in) return hipSuccess;
  hipLaunchKernelGGL(join_columns_kernel, dim3((unsigned)((p.d + 15) / 16), 2), dim3(256), 0, st, p.part, n, p.d, p.w_out,
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
