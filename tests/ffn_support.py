"""Plain 64-bit forms of the operators of include/omnimoe_ffn.h and bounds on what the kernels' rounding may change.

A bound is first order, element by element: a sum of n products in fp32 is within 2 n 2^-24 of the sum of their
magnitudes (Higham, Thm 3.1, twice), a value rounded to bf16 within 2^-8 of itself, and errors pass through products and
through silu (|silu'| <= 1.1, |silu''| <= 0.5) as their derivatives say. Four units of 2^-24 stand for each elementwise
formula's own roundings (exp, division and products).
"""
from __future__ import annotations

from types import SimpleNamespace

import torch

import paper_2602_05711_amd as P

U32 = 2.0 ** -24
F64 = torch.float64


def unit(dtype):
    """Half a step of the type, relative."""
    return torch.finfo(dtype).eps / 2


def gamma(n):
    return 2 * n * U32


def desc(T, d, dtype, **kw):
    f = dict(n_rows=16, n_cols=16, d_key=8, H=1, K=1, act="gelu", query_mode="split" if d >= 16 else "shared",
             group_size=1)
    f.update(kw)
    return P.make_desc(SimpleNamespace(T=T, d=d, dtype="bf16" if dtype is torch.bfloat16 else "f32", **f))


def randn(seed, *shape, scale=1.0, dtype=torch.float32, device="cuda"):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).to(device)


def silu(g):
    return g / (1 + torch.exp(-g))


def dsilu(g):
    s = 1 / (1 + torch.exp(-g))
    return s * (1 + g * (1 - s))


# ------------------------------------------------------------------ checkpoint

def quantise(x):
    """(values, scale bytes) of x [T, d] in 64 bits, by the definition of e4m3: three bits after the leading one, the
    least exponent -6, the even neighbour where two are as near; values that are not finite come back as NaN."""
    x = x.to(F64)
    T, d = x.shape
    nb = -(-d // 32)
    b = torch.zeros((T, nb * 32), dtype=F64, device=x.device)
    b[:, :d] = x
    b = b.view(T, nb, 32)
    fine = torch.isfinite(b)
    most = torch.where(fine, b.abs(), 0.0).amax(-1, keepdim=True)
    s = torch.full_like(most, -127.0)
    for e in range(-126, 121):
        s = torch.where(most > 448.0 * 2.0 ** (e - 1), float(e), s)
    v = torch.where(fine, b, 0.0) * torch.exp2(-s)
    m, ex = torch.frexp(v)  # v = m 2^ex, 1/2 <= |m| < 1: the leading bit is 2^(ex - 1)
    step = torch.exp2((ex - 1).clamp(min=-6).to(F64) - 3)
    q = torch.round(v / step) * step * torch.exp2(s)
    q = torch.where(fine, q, float("nan"))
    return q.view(T, -1)[:, :d], (s.view(T, nb) + 127).to(torch.uint8)


def dequantise(codes, scales):
    byte = codes.long()
    e, m = (byte >> 3) & 15, (byte & 7).to(F64)
    v = torch.where(e > 0, (8 + m) * torch.exp2(e.to(F64) - 10), m * 2.0 ** -9)
    v = torch.where((byte & 127) == 127, float("nan"), v)
    v = torch.where(byte > 127, -v, v)
    block = torch.arange(codes.shape[1], device=codes.device) // 32
    return v * torch.exp2(scales.to(F64)[:, block] - 127)


# ------------------------------------------------------------------ the shared branch's way back

def mlp_backward(x, w_gu, w_down, dy):
    """(dx, dw_gu, dw_down) in 64 bits for inputs in 64 bits."""
    f = w_down.shape[1]
    h = x @ w_gu.t()
    g, u = h[:, :f], h[:, f:]
    da = dy @ w_down
    dh = torch.cat((da * u * dsilu(g), da * silu(g)), 1)
    return dh @ w_gu, dh.t() @ x, dy.t() @ (silu(g) * u)


def mlp_backward_bounds(x, w_gu, w_down, dy, dx_in, dtype):
    T, d = x.shape
    f = w_down.shape[1]
    r = unit(dtype) if dtype is torch.bfloat16 else 0.0  # the operands' rounding
    h, eh = x @ w_gu.t(), gamma(d) * (x.abs() @ w_gu.abs().t())
    g, u, eg, eu = h[:, :f], h[:, f:], eh[:, :f], eh[:, f:]
    da = dy @ w_down
    # dy as two bf16 values: 2^-8 of 2^-8 is left
    eda = (gamma(2 * d) + r * r) * (dy.abs() @ w_down.abs())
    dg, du, a = da * u * dsilu(g), da * silu(g), silu(g) * u
    edg = eda * u.abs() * 1.1 + da.abs() * (1.1 * eu + 0.5 * u.abs() * eg) + 4 * U32 * (da * u).abs()
    edu = eda * silu(g).abs() + da.abs() * 1.1 * eg + 4 * U32 * du.abs()
    ea = 1.1 * eg * u.abs() + silu(g).abs() * eu + 4 * U32 * a.abs()
    dh = torch.cat((dg, du), 1)
    edh = torch.cat((edg, edu), 1) + r * dh.abs()
    ea = ea + r * a.abs()
    dx, dwg, dwd = dh @ w_gu + dx_in, dh.t() @ x, dy.t() @ a
    last = unit(dtype)
    bx = edh @ w_gu.abs() + gamma(2 * f + 1) * (dh.abs() @ w_gu.abs() + dx_in.abs()) + last * dx.abs()
    bg = edh.t() @ x.abs() + gamma(T + 64) * (dh.abs().t() @ x.abs()) + last * dwg.abs()
    bd = dy.abs().t() @ ea + (gamma(2 * T + 64) + r * r) * (dy.abs().t() @ a.abs()) + last * dwd.abs()
    return (dx, dwg, dwd), (bx, bg, bd)


# ------------------------------------------------------------------ adapters

def adapters_mlp(x, w_gu, w_down, ids, tables, y_in, dtype):
    """(y, bound) in 64 bits; tables: a_gu, b_gu, a_down, b_down, scale."""
    T, d = x.shape
    f = w_down.shape[1]
    a_gu, b_gu, a_down, b_down, scale = tables
    n, rank = a_down.shape[:2]
    bf16 = dtype is torch.bfloat16
    r = unit(dtype) if bf16 else 0.0
    rl = r if T > 64 else 0.0  # the rank-wide values' rounding
    h, eh = x @ w_gu.t(), gamma(d) * (x.abs() @ w_gu.abs().t())
    rows = [(e, (ids == e).nonzero().flatten()) for e in range(n)]
    rows = [(e, at) for e, at in rows if at.numel()]
    for e, at in rows:
        A, Bm, s = a_gu[e].to(F64), b_gu[e].to(F64), float(scale[e])
        low = s * (x[at] @ A.t())
        el = (gamma(d) + 2 * U32) * abs(s) * (x[at].abs() @ A.abs().t()) + rl * low.abs()
        for part in (0, 1):
            B_, l_, e_ = Bm[part * f:(part + 1) * f], low[:, part * rank:(part + 1) * rank], el[:, part * rank:(part + 1) * rank]
            h[at, part * f:(part + 1) * f] += l_ @ B_.t()
            eh[at, part * f:(part + 1) * f] += e_ @ B_.abs().t() + gamma(rank + 1) * (l_.abs() @ B_.abs().t())
    eh += 2 * U32 * h.abs()
    g, u, eg, eu = h[:, :f], h[:, f:], eh[:, :f], eh[:, f:]
    a = silu(g) * u
    ea = 1.1 * eg * u.abs() + silu(g).abs() * eu + (4 * U32 + r) * a.abs()
    y = y_in + a @ w_down.t()
    ey = ea @ w_down.abs().t() + gamma(f + 2) * (a.abs() @ w_down.abs().t() + y_in.abs())
    for e, at in rows:
        A, Bm, s = a_down[e].to(F64), b_down[e].to(F64), float(scale[e])
        low = s * (a[at] @ A.t())
        el = abs(s) * (ea[at] @ A.abs().t() + (gamma(f) + 2 * U32) * (a[at].abs() @ A.abs().t())) + rl * low.abs()
        y[at] += low @ Bm.t()
        ey[at] += el @ Bm.abs().t() + gamma(rank + 1) * (low.abs() @ Bm.abs().t())
    return y, ey + (unit(dtype) + 2 * U32) * y.abs()


# ------------------------------------------------------------------ the layer for a few tokens

def steps(seed, *shape, scale, step, dtype):
    """Gaussian values in whole multiples of `step` (at most 256 of them): products of two such tensors sum exactly in
    fp32 in any order, so that logits, and the selection with them, do not depend on it."""
    g = torch.Generator().manual_seed(seed)
    v = (torch.randn(shape, generator=g) * (scale / step)).round().clamp(-256, 256) * step
    return v.to(dtype).cuda()


def few_layer(x, keys_row, keys_col, u, v, w_gu, w_down, K, act, split):
    """(idx, gates, y, bound of y) in 64 bits; equal scores go to the lower id."""
    T, d = x.shape
    H, nr, dk = keys_row.shape
    nc = keys_col.shape[1]
    X = x.to(F64)
    xr, xc = X[:, :dk], X[:, dk:2 * dk] if split else X[:, :dk]
    idx = torch.empty((T, H, K), dtype=torch.int64, device=x.device)
    gates = torch.empty((T, H, K), dtype=F64, device=x.device)
    y = torch.zeros((T, d), dtype=F64, device=x.device)
    ey = torch.zeros_like(y)
    mag = torch.zeros_like(y)
    for t in range(T):
        for h in range(H):
            grid = ((keys_row[h].to(F64) @ xr[t])[:, None] + keys_col[h].to(F64) @ xc[t]).flatten()
            at = torch.sort(grid, descending=True, stable=True).indices[:K]
            idx[t, h] = at
            gates[t, h] = g = torch.softmax(grid[at], 0)
            U, V = u[at].to(F64), v[at].to(F64)
            z = U @ X[t]
            ez = gamma(d) * (U.abs() @ X[t].abs())
            a = silu(z) if act == "silu" else 0.5 * z * torch.erfc(-z * 0.5 ** 0.5)
            w, ew = g * a, g * 1.13 * ez + (K + 16) * U32 * g * (a.abs() + z.abs() * 2.0 ** -3)
            y[t] += w @ V
            ey[t] += ew @ V.abs()
            mag[t] += w.abs() @ V.abs()
    ey += gamma(K + H) * mag
    if w_gu is not None:
        f = w_down.shape[1]
        G, D = w_gu.to(F64), w_down.to(F64)
        hid, eh = X @ G.t(), gamma(d) * (X.abs() @ G.abs().t())
        g, uu = hid[:, :f], hid[:, f:]
        a = silu(g) * uu
        ea = 1.1 * eh[:, :f] * uu.abs() + silu(g).abs() * eh[:, f:] + 4 * U32 * a.abs()
        y += a @ D.t()
        # (three bf16 values hold a to 2^-24)
        ey += ea @ D.abs().t() + (gamma(3 * f) + 2 * U32) * (a.abs() @ D.abs().t())
    return idx, gates, y, ey + 2 * U32 * y.abs() + gamma(2) * mag
