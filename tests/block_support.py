"""Plain 64-bit forms of the operators of include/omnimoe_block.h and bounds on what the kernels' rounding may change.

Bounds are first order, element by element, as in ffn_support: a sum of n products in fp32 is within 2 n 2^-24 of the sum of
their magnitudes, a result rounded to the layer's type within half a step of itself. A norm's factor 1 / sqrt(mean v^2 +
eps) comes from a sum of d squares, none negative, so that its relative error is half of d 2^-24 and a few roundings
(`norm_err`); sigmoid(g) and 1 - sigmoid(g) are within six units of themselves (exp two, a sum and a division).
"""
from __future__ import annotations

import torch

from ffn_support import F64, U32, gamma, silu, unit

SIG = 6 * U32


def norm_err(d):
    return (d / 2 + 8) * U32


def least(dtype):
    """Half a step of the type's subnormal values, which a rounding is off by where relative steps end, with the same of two
    fp32 values on the way: 2^-134 and 2^-149 for bf16 (least value 2^-133), 2^-150 and 2^-149 for fp32 (2^-149)."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2 + 2.0 ** -149


# ------------------------------------------------------------------ the joint

def join(x, y, gate, w_out, scale, w_in, eps):
    """(x_out, n) in 64 bits; any of y, gate, w_out, scale, w_in may be None; gate [T, 1] or [T, d]."""
    z = x
    if y is not None:
        b = y if w_out is None else w_out * y / torch.sqrt((y * y).mean(1, keepdim=True) + eps)
        if gate is not None:
            b = b / (1 + torch.exp(-gate))
        z = x + (b if scale is None else scale * b)
    n = None if w_in is None else w_in * z / torch.sqrt((z * z).mean(1, keepdim=True) + eps)
    return z, n


def join_bounds(x, y, gate, w_out, scale, w_in, eps, dtype):
    d, r = x.shape[1], unit(dtype)
    z, n = join(x, y, gate, w_out, scale, w_in, eps)
    e = torch.zeros_like(x)
    if y is not None:
        e = (z - x).abs() * (norm_err(d) + SIG + 8 * U32) + 2 * U32 * z.abs()
    ez = e * (1 + r) + r * z.abs()
    if n is None:
        return (z, n), (ez, None)
    rho = 1 / torch.sqrt((z * z).mean(1, keepdim=True) + eps)
    rel = rho * rho * (z.abs() * e).mean(1, keepdim=True) + norm_err(d) + 6 * U32
    return (z, n), (ez, (1 + r) * (w_in.abs() * rho * e + rel * n.abs()) + r * n.abs())


def join_back(x, y, gate, w_out, scale, w_in, dx_out, dn, eps):
    """dict of the gradients in 64 bits, from the formulas; x is x_out."""
    T, d = x.shape
    G = torch.zeros_like(x) if dx_out is None else dx_out
    out = {}
    if w_in is not None:
        rho = 1 / torch.sqrt((x * x).mean(1, keepdim=True) + eps)
        xh, u = x * rho, dn * w_in
        G = G + rho * (u - xh * (u * xh).mean(1, keepdim=True))
        out["dw_in"] = (dn * xh).sum(0)
    out["dx"] = G
    if y is None:
        return out
    r = 1.0 if w_out is None else 1 / torch.sqrt((y * y).mean(1, keepdim=True) + eps)
    yh = y * r
    s = 1.0 if gate is None else 1 / (1 + torch.exp(-gate))
    a = (1.0 if scale is None else scale) * (1.0 if w_out is None else w_out) * torch.ones(d, dtype=F64, device=x.device)
    q = G * s * a
    out["dy"] = r * (q - yh * (q * yh).mean(1, keepdim=True)) if w_out is not None else q
    S = (G * s * yh).sum(0)
    if w_out is not None:
        out["dw_out"] = S if scale is None else scale * S
    if scale is not None:
        out["dscale"] = S if w_out is None else w_out * S
    if gate is not None:
        g = q * yh / (1 + torch.exp(gate))
        out["dgate"] = g.sum(1, keepdim=True) if gate.shape[1] == 1 else g
    return out


def join_back_bounds(x, y, gate, w_out, scale, w_in, dx_out, dn, eps, dtype):
    T, d = x.shape
    r_ = unit(dtype)
    want = join_back(x, y, gate, w_out, scale, w_in, dx_out, dn, eps)
    ne, b = norm_err(d), {}
    G = want["dx"]
    eG = 2 * U32 * G.abs()
    if w_in is not None:
        rho = 1 / torch.sqrt((x * x).mean(1, keepdim=True) + eps)
        xh, u = x * rho, dn * w_in
        m = (u * xh).mean(1, keepdim=True)
        em = (gamma(d) + ne + 4 * U32) * (u * xh).abs().mean(1, keepdim=True)
        eG = eG + rho * (u.abs() * (ne + 4 * U32) + xh.abs() * (m.abs() * (2 * ne + 4 * U32) + em))
        eG = eG + 2 * U32 * (rho * (u.abs() + (xh * m).abs()) + (0 if dx_out is None else dx_out.abs()))
        b["dw_in"] = (gamma(T + 64) + ne + 4 * U32) * (dn * xh).abs().sum(0)
    b["dx"] = (1 + r_) * eG + r_ * G.abs() + least(dtype)
    if y is None:
        return want, b
    r = 1.0 if w_out is None else 1 / torch.sqrt((y * y).mean(1, keepdim=True) + eps)
    ye = U32 if w_out is None else ne
    yh = y * r
    s = torch.ones((), dtype=F64, device=x.device) if gate is None else 1 / (1 + torch.exp(-gate))
    a = ((1.0 if scale is None else scale) * (1.0 if w_out is None else w_out) * torch.ones(d, dtype=F64, device=x.device)).abs()
    q = (G * s).abs() * a
    eq = s * a * eG + q * (SIG + 6 * U32)
    m2, em2 = (G * s * a * yh).abs().mean(1, keepdim=True), 0
    em2 = (eq * yh.abs() + (q * yh).abs() * (ye + gamma(d) + 2 * U32)).mean(1, keepdim=True)
    b["dy"] = r * eq + (r * q) * (ye + 4 * U32) + least(torch.float32)
    if w_out is not None:
        b["dy"] = b["dy"] + r * (yh.abs() * em2 + (yh * m2).abs() * (2 * ye + 8 * U32))
    Ss = (eG * s * yh.abs() + (G * s * yh).abs() * (ye + SIG + 6 * U32 + gamma(T + 64))).sum(0)
    if w_out is not None:
        b["dw_out"] = (1.0 if scale is None else scale.abs()) * Ss + 2 * U32 * want["dw_out"].abs()
    if scale is not None:
        b["dscale"] = (1.0 if w_out is None else w_out.abs()) * Ss + 2 * U32 * want["dscale"].abs()
    if gate is not None:
        o = 1 / (1 + torch.exp(gate))
        if gate.shape[1] == 1:
            e = o * (em2 * d) + (SIG + 4 * U32) * o * m2 * d
        else:
            e = o * (eq * yh.abs() + (q * yh).abs() * (ye + SIG + 6 * U32))
        b["dgate"] = (1 + r_) * e + r_ * want["dgate"].abs() + least(dtype)
    return want, b


# ------------------------------------------------------------------ products grouped by expert

def schedule(idx, N):
    """(perm, offsets) of a flat list of expert ids: the stable order by expert."""
    perm = torch.sort(idx.long(), stable=True).indices
    offsets = torch.zeros(N + 1, dtype=torch.int64, device=idx.device)
    offsets[1:] = torch.bincount(idx.long(), minlength=N).cumsum(0)
    return perm.to(torch.int32), offsets.to(torch.int32)


def rows_of(perm, order, hk, M, device):
    if order == "position":
        return torch.arange(M, device=device)
    return perm.long() // (hk if order == "token" else 1)


def product(x, w, offsets, swiglu, dtype):
    """(y by position, its bound) in 64 bits for x by position; rows past offsets[-1] are zeros."""
    M, k = x.shape
    n = w.shape[1] // (2 if swiglu else 1)
    y = torch.zeros((M, n), dtype=F64, device=x.device)
    e = torch.zeros_like(y)
    ends = offsets.tolist()
    for i, (lo, hi) in enumerate(zip(ends[:-1], ends[1:])):
        if hi <= lo:
            continue
        X, W = x[lo:hi], w[i].to(F64)
        h, eh = X @ W.t(), gamma(k) * (X.abs() @ W.abs().t())
        if swiglu:
            g, u, eg, eu = h[:, :n], h[:, n:], eh[:, :n], eh[:, n:]
            y[lo:hi] = silu(g) * u
            e[lo:hi] = 1.1 * eg * u.abs() + silu(g).abs() * eu + 8 * U32 * (silu(g) * u).abs()
        else:
            y[lo:hi], e[lo:hi] = h, eh
    r = unit(dtype)
    return y, e * (1 + r) + r * y.abs()


def product_dw(x, dy, offsets, dtype):
    """(dw, its bound) in 64 bits for rows by position."""
    ends, r = offsets.tolist(), unit(dtype)
    dw, e = [], []
    for lo, hi in zip(ends[:-1], ends[1:]):
        X, D = x[lo:max(lo, hi)], dy[lo:max(lo, hi)]
        v = D.t() @ X
        dw.append(v)
        e.append((1 + r) * gamma(hi - lo + 64) * (D.abs().t() @ X.abs()) + r * v.abs())
    return torch.stack(dw), torch.stack(e)


def product_dx(dy, w, offsets, dtype):
    y, e = product(dy, w.transpose(1, 2), offsets, False, dtype)
    return y, e


# ------------------------------------------------------------------ 4-bit weights

LIST4 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def quantise4(w):
    """(values, scale bytes) of the rows' blocks of 32 in 64 bits, by the definition."""
    w = w.to(F64)
    b = w.reshape(-1, 32)
    fine = torch.isfinite(b).all(1, keepdim=True)
    b = torch.where(torch.isfinite(b), b, 0.0)
    most = b.abs().amax(1, keepdim=True)
    s = torch.full_like(most, -125.0)
    for e in range(-124, 126):
        s = torch.where(most > 6.0 * 2.0 ** (e - 1), float(e), s)
    v = (b * torch.exp2(-s)).unsqueeze(-1)
    place = torch.tensor(LIST4, dtype=F64, device=w.device)
    off = (v.abs() - place).abs()
    near = off.amin(-1, keepdim=True)
    both = off == near  # one place, or two neighbours: the even one
    even = torch.arange(8, device=w.device) % 2 == 0
    pick = torch.where(both.sum(-1, keepdim=True) == 2, both & even, both)
    q = (pick * place).sum(-1) * torch.sign(v[..., 0]) * torch.exp2(s)
    q = torch.where(fine, q, float("nan"))
    byte = torch.where(fine, s + 127, 255.0).to(torch.uint8)
    return q.view(w.shape), byte.view(*w.shape[:-1], w.shape[-1] // 32)


def dequantise4(codes, scales):
    q = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    v = torch.tensor(LIST4, dtype=F64, device=codes.device)[q & 7]
    v = torch.where(q > 7, -v, v).view(*scales.shape, 32)
    v = v * torch.exp2(scales.to(F64) - 127).unsqueeze(-1)
    return torch.where(scales.unsqueeze(-1) == 255, float("nan"), v).flatten(-2)


