"""What is measured of the block around the layer and of routed experts with matrices of their own: the norms, gate and
residual scale that join a branch to the residual stream, with their gradients; the matrix products of rows grouped by
expert, with their gradients; and the same products with 4-bit weights.

A case is a dict of plain values. Its ``mode`` is the call that a program makes:

* ``join``        omnimoe_block_join: x' = x + scale * sigmoid(gate) * norm(y) and n = norm(x'), the next layer's input;
* ``join_back``   omnimoe_block_join_backward: gradients of all of its inputs;
* ``product``     omnimoe_grouped_product: y_p = W_e x_p for the rows p of every expert e, or the SwiGLU of gate and up
                  rows;
* ``product_back``  omnimoe_grouped_product_dx and omnimoe_grouped_product_dw;
* ``product4``    omnimoe_grouped_product4: the product with weights held in 4 bits.

``listed()`` names the cases, ``draw(rng)`` gives others of the same ranges, ``prepare`` makes what the program holds
before the call, ``run`` makes the call (or, where ``own`` is false, computes the same in plain torch) and ``exact``
recomputes the outputs in 64 bits.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import torch

own = False

EPS = 1e-6


def listed():
    return [
        # One decoded token, whose time is a launch's; the training batch with a gate for every token.
        dict(name="join_token", mode="join", T=1, d=2048, gate="token", dtype="bf16"),
        dict(name="join_train", mode="join", T=16384, d=2048, gate="token", dtype="bf16"),
        # The way back: the fp32 layer of accuracy work, and the training batch with a gate for every channel.
        dict(name="join_back_f32", mode="join_back", T=1000, d=520, gate="channel", dtype="f32"),
        dict(name="join_back_train", mode="join_back", T=16384, d=2048, gate="channel", dtype="bf16"),
        # Gate and up projection of 64 experts: a decode step of sixteen tokens, whose time is the weights', and the
        # training batch. A ragged fp32 batch on twelve experts, results in task order.
        dict(name="product_decode16", mode="product", T=16, K=8, rows=8, cols=8, n_in=2048, n_out=1024, swiglu=True,
             x_order="token", y_order="position", dtype="bf16"),
        dict(name="product_f32", mode="product", T=333, K=4, rows=3, cols=4, n_in=520, n_out=264, swiglu=False,
             x_order="position", y_order="task", dtype="f32"),
        dict(name="product_train", mode="product", T=16384, K=8, rows=8, cols=8, n_in=2048, n_out=1024, swiglu=True,
             x_order="token", y_order="position", dtype="bf16"),
        # The way back through a small model's experts and through those of the training layer.
        dict(name="product_back_small", mode="product_back", T=1021, K=2, rows=4, cols=4, n_in=512, n_out=512,
             x_order="token", y_order="position", dtype="bf16"),
        dict(name="product_back_train", mode="product_back", T=8192, K=8, rows=8, cols=8, n_in=2048, n_out=2048,
             x_order="token", y_order="position", dtype="bf16"),
        # 4-bit experts: one decoded token and a decode step of sixteen; one fp32 matrix, as a shared branch has it.
        dict(name="product4_decode1", mode="product4", T=1, K=8, rows=8, cols=8, n_in=2048, n_out=1024, swiglu=True,
             x_order="token", y_order="position", dtype="bf16"),
        dict(name="product4_decode16", mode="product4", T=16, K=8, rows=8, cols=8, n_in=2048, n_out=1024, swiglu=True,
             x_order="token", y_order="position", dtype="bf16"),
        dict(name="product4_f32", mode="product4", T=7, K=1, rows=1, cols=1, n_in=2080, n_out=2056, swiglu=False,
             x_order="position", y_order="position", dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any of the modes, one token to the training batch, odd lengths and widths (multiples of 8, of 32
    where blocks of 4-bit weights ask for it) among them."""
    mode = rng.choice(["join", "join_back", "product", "product", "product_back", "product4", "product4"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if mode in ("join", "join_back"):
        d = rng.choice([8 * _log_int(rng, 2, 512), 512, 1024, 2048])
        if dtype == "f32":
            d = min(d, 2048)
        return dict(mode=mode, T=_log_int(rng, 1, min(16384, (1 << 25) // d)), d=d,
                    gate=rng.choice(["none", "token", "channel"]), dtype=dtype)
    rows, cols = rng.choice([(1, 1), (2, 2), (3, 4), (4, 4), (4, 8), (8, 8), (8, 8), (8, 16), (16, 16)])
    N = rows * cols
    K = rng.randint(1, min(N, 8))
    if mode == "product4":
        n_in, n_out = 32 * _log_int(rng, 2, 64), 8 * _log_int(rng, 8, 256)
        T, limit = _log_int(rng, 1, 64), 1 << 28
    else:
        n_in = rng.choice([8 * _log_int(rng, 8, 256), 512, 1024, 2048])
        n_out = rng.choice([8 * _log_int(rng, 8, 256), 512, 1024, 2048])
        T = _log_int(rng, 1, 16384) if mode == "product" else _log_int(rng, 16, 8192)
        limit = 1 << 28
    if dtype == "f32":
        n_in, n_out, T = min(n_in, 1024), min(n_out, 1024), min(T, 1024)
    while N * n_in * n_out > limit:
        n_out = max(64, n_out // 16 * 8)
        if n_out == 64:
            break
    T = max(1, min(T, (1 << 38) // (K * n_in * n_out)))
    orders = [("token", "position"), ("position", "task"), ("position", "position"), ("task", "task")]
    x_order, y_order = rng.choice(orders)
    case = dict(mode=mode, T=T, K=K, rows=rows, cols=cols, n_in=n_in, n_out=n_out, x_order=x_order, y_order=y_order,
                dtype=dtype)
    if mode != "product_back":
        case["swiglu"] = rng.random() < 0.5
    return case


# ------------------------------------------------------------------ inputs

def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _normal(case, seed, stream, shape, scale=1.0, dtype=None):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 32 + stream)
    t = torch.randn(shape, generator=g, device="cuda", dtype=dtype or _type(case))
    return t.mul_(scale) if scale != 1.0 else t


def _join_tensors(case, seed):
    T, d, f32 = case["T"], case["d"], torch.float32
    # channels of very different size, as a residual stream has them
    wide = torch.exp2(1.5 * _normal(case, seed, 2, (d,), 1.0, f32)).to(_type(case))
    t = dict(x=_normal(case, seed, 1, (T, d)).mul_(wide), y=_normal(case, seed, 3, (T, d), 0.2, f32),
             gate=None, w_out=_normal(case, seed, 4, (d,), 0.1, f32).add_(1.0),
             scale=_normal(case, seed, 5, (d,), 0.05, f32).add_(0.5), w_in=_normal(case, seed, 6, (d,), 0.1, f32).add_(1.0))
    if case["gate"] != "none":
        t["gate"] = _normal(case, seed, 7, (T, 1 if case["gate"] == "token" else d))
    if case["mode"] == "join_back":  # x is the stream behind the join; gradients of a loss averaged over the tokens
        t["dx_out"] = _normal(case, seed, 8, (T, d), 1.0 / T)
        t["dn"] = _normal(case, seed, 9, (T, d), 1.0 / T)
    return t


def _schedule(case, seed):
    """Every token's K experts (some are more popular than others), and the tasks in the experts' order: perm [T K],
    offsets [N + 1], as omnimoe_schedule gives them."""
    T, K, N = case["T"], case["K"], case["rows"] * case["cols"]
    liked = _normal(case, seed, 10, (1, N), 0.4, torch.float32)
    idx = torch.topk(_normal(case, seed, 11, (T, N), 1.0, torch.float32) + liked, K, dim=1).indices.flatten()
    perm = torch.sort(idx, stable=True).indices.to(torch.int32)
    offsets = torch.zeros((N + 1,), dtype=torch.int32, device="cuda")
    offsets[1:] = torch.bincount(idx, minlength=N).cumsum(0)
    return perm, offsets


def _product_tensors(case, seed):
    c = SimpleNamespace(swiglu=case.get("swiglu", False), **{k: v for k, v in case.items() if k != "swiglu"})
    N, M = c.rows * c.cols, c.T * c.K
    perm, offsets = _schedule(case, seed)
    t = dict(perm=perm, offsets=offsets, x=_normal(case, seed, 1, (c.T if c.x_order == "token" else M, c.n_in)))
    w = _normal(case, seed, 2, (N, (2 if c.swiglu else 1) * c.n_out, c.n_in), 1.0 / math.sqrt(c.n_in))
    if c.mode == "product4":
        t["codes"], t["scales"] = _quantise4(w)
    else:
        t["w"] = w
    if c.mode == "product_back":
        t["dy"] = _normal(case, seed, 3, (M, c.n_out), 1.0 / c.T)
    return t


def _quantise4(w):
    """(codes, scale bytes) of the rows' blocks of 32: the scale is the least power of two that brings the block's largest
    magnitude to 6 or below; its byte is the exponent plus 127. Two codes a byte, the first in the low bits: a sign bit
    and the place in 0, 0.5, 1, 1.5, 2, 3, 4, 6."""
    N, n, k = w.shape
    b = w.float().view(N, n, k // 32, 32)
    m, e = torch.frexp(b.abs().amax(-1))
    s = torch.where(m > 0, e - 3 + (m > 0.75), -125).clamp_(-125, 125)
    v = b / torch.exp2(s.float())[..., None]
    ends = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=w.device)
    even = torch.tensor([1, 3, 5], device=w.device)  # (the borders whose tie goes up, to the even code)
    a = v.abs().contiguous()
    code = torch.bucketize(a, ends) + (a[..., None] == ends[even]).any(-1)
    code = (code + 8 * (v < 0)).to(torch.uint8).view(N, n, k // 2, 2)
    return code[..., 0] | (code[..., 1] << 4), (s + 127).to(torch.uint8)


def prepare(case, seed):
    if case["mode"] in ("join", "join_back"):
        return SimpleNamespace(case=dict(case), kept=None, **_join_tensors(case, seed))
    t = _product_tensors(case, seed)
    # the longest expert's rows: what a program that pads its experts to one length plans with
    most = int((t["offsets"][1:] - t["offsets"][:-1]).max())
    return SimpleNamespace(case=dict(case), kept=None, most=most, **t)


# ------------------------------------------------------------------ the plain forms

def _plain_join(s):
    y = s.y
    b = s.w_out * (y * torch.rsqrt((y * y).mean(1, keepdim=True) + EPS))
    if s.gate is not None:
        b = torch.sigmoid(s.gate.float()) * b
    x = s.x.float() + s.scale * b
    n = s.w_in * (x * torch.rsqrt((x * x).mean(1, keepdim=True) + EPS))
    return dict(x_out=x.to(s.x.dtype), n=n.to(s.x.dtype))


def _plain_join_back(s):
    x, y, dn, dt = s.x.float(), s.y, s.dn.float(), s.x.dtype
    rho = torch.rsqrt((x * x).mean(1, keepdim=True) + EPS)
    xh = x * rho
    u = dn * s.w_in
    g = s.dx_out.float() + rho * (u - xh * (u * xh).mean(1, keepdim=True))
    r = torch.rsqrt((y * y).mean(1, keepdim=True) + EPS)
    yh = y * r
    p = torch.sigmoid(s.gate.float()) if s.gate is not None else torch.ones((), device=x.device)
    total = (g * p * yh).sum(0)
    q = g * p * (s.scale * s.w_out)
    out = dict(dx=g.to(dt), dy=r * (q - yh * (q * yh).mean(1, keepdim=True)), dw_in=(dn * xh).sum(0),
               dw_out=s.scale * total, dscale=s.w_out * total)
    if s.gate is not None:
        dp = g * (s.scale * s.w_out) * yh
        out["dgate"] = ((dp.sum(1, keepdim=True) if s.gate.shape[1] == 1 else dp) * p * (1 - p)).to(dt)
    return out


def _places(s):
    """Each position's expert and its place among that expert's rows."""
    at = torch.arange(s.perm.numel(), device="cuda")
    e = torch.searchsorted(s.offsets[1:].contiguous(), at.to(torch.int32), right=True)
    return e, at - s.offsets.long()[e]


def _padded(s, rows, e, at):
    p = torch.zeros((s.offsets.numel() - 1, s.most, rows.shape[1]), device="cuda")
    p[e, at] = rows
    return p


def _in_order(s, t, order):
    """The rows of t, which lie by position, by task or by token, by position."""
    if order == "position":
        return t
    return t[s.perm.long() // (s.case["K"] if order == "token" else 1)]


def _from_positions(s, rows, order):
    if order == "position":
        return rows
    out = torch.empty_like(rows)
    out[s.perm.long()] = rows
    return out


def _plain_product(s):
    c = s.case
    if c["mode"] == "product4":
        value = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device="cuda")
        code = torch.stack((s.codes & 15, s.codes >> 4), -1).flatten(2).int()
        w = torch.where(code > 7, -value[code & 7], value[code & 7])
        w = (w.view(*s.scales.shape, 32) * torch.exp2(s.scales.float() - 127)[..., None]).flatten(2)
    else:
        w = s.w.float()
    e, at = _places(s)
    h = torch.bmm(_padded(s, _in_order(s, s.x, c["x_order"]).float(), e, at), w.transpose(1, 2))[e, at]
    if c["swiglu"]:
        g, u = h.chunk(2, 1)
        h = g * torch.sigmoid(g) * u
    return dict(y=_from_positions(s, h.to(s.x.dtype), c["y_order"]))


def _plain_product_back(s):
    c = s.case
    e, at = _places(s)
    x = _padded(s, _in_order(s, s.x, c["x_order"]).float(), e, at)
    dy = _padded(s, _in_order(s, s.dy, c["y_order"]).float(), e, at)
    dx = torch.bmm(dy, s.w.float())[e, at].to(s.x.dtype)
    # (a token's rows come back one a task: the program adds them with the gates' gradients)
    return dict(dx=_from_positions(s, dx, _dx_order(c)), dw=torch.bmm(dy.transpose(1, 2), x).to(s.x.dtype))


def _dx_order(c):
    return "task" if c["x_order"] == "token" else c["x_order"]


# ------------------------------------------------------------------ the framework's calls

def _kept(s):
    """Descriptors, outputs and workspace, made at the first pass and kept, as a program does."""
    import paper_2602_05711_amd as P
    c = s.case
    k = SimpleNamespace(P=P)

    def new(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda")

    join = c["mode"] in ("join", "join_back")
    d = c["d"] if join else 64  # (the products' widths are their own)
    k.desc = P.make_desc(SimpleNamespace(T=c["T"], d=d, n_rows=c.get("rows", 1), n_cols=c.get("cols", 1), d_key=8, H=1,
                                         K=c.get("K", 1), dtype=c["dtype"], query_mode="shared"))
    if join:
        T, dt, f32 = c["T"], s.x.dtype, torch.float32
        if c["mode"] == "join":
            k.x_out, k.n = new((T, d), dt), new((T, d), dt)
        else:
            k.dx, k.dy, k.dgate = new((T, d), dt), new((T, d), f32), None if s.gate is None else torch.empty_like(s.gate)
            k.dw_out, k.dscale, k.dw_in = new((d,), f32), new((d,), f32), new((d,), f32)
            k.ws = new((max(256, P.omnimoe_block_join_backward_workspace_size(k.desc)),), torch.uint8)
        return k
    M = c["T"] * c["K"]

    def product(x_order):
        return P.make_product(c["n_in"], c["n_out"], swiglu=c.get("swiglu", False), x_order=x_order, y_order=c["y_order"])

    k.product = product(c["x_order"])
    if c["mode"] == "product_back":
        k.product_dx = product(_dx_order(c))
        k.dx, k.dw = new((M, c["n_in"]), s.x.dtype), torch.empty_like(s.w)
        k.ws = new((max(256, P.omnimoe_grouped_product_dw_workspace_size(k.desc, k.product)),), torch.uint8)
    else:
        k.y = new((M, c["n_out"]), s.x.dtype)
    return k


def run(s):
    mode = s.case["mode"]
    if not own:
        return {"join": _plain_join, "join_back": _plain_join_back, "product": _plain_product, "product4": _plain_product,
                "product_back": _plain_product_back}[mode](s)
    if s.kept is None:
        s.kept = _kept(s)
    k = s.kept
    if mode == "join":
        k.P.omnimoe_block_join(k.desc, EPS, s.x, s.y, s.gate, s.w_out, s.scale, s.w_in, k.x_out, k.n)
        return dict(x_out=k.x_out, n=k.n)
    if mode == "join_back":
        k.P.omnimoe_block_join_backward(k.desc, EPS, s.x, s.y, s.gate, s.w_out, s.scale, s.w_in, s.dx_out, s.dn, k.dx,
                                        k.dy, k.dgate, k.dw_out, k.dscale, k.dw_in, ws=k.ws)
        out = dict(dx=k.dx, dy=k.dy, dw_in=k.dw_in, dw_out=k.dw_out, dscale=k.dscale)
        return out if s.gate is None else dict(out, dgate=k.dgate)
    if mode == "product":
        k.P.omnimoe_grouped_product(k.desc, k.product, s.x, s.w, s.offsets, s.perm, k.y)
        return dict(y=k.y)
    if mode == "product4":
        k.P.omnimoe_grouped_product4(k.desc, k.product, s.x, s.codes, s.scales, s.offsets, s.perm, k.y)
        return dict(y=k.y)
    k.P.omnimoe_grouped_product_dx(k.desc, k.product_dx, s.dy, s.w, s.offsets, s.perm, k.dx)
    k.P.omnimoe_grouped_product_dw(k.desc, k.product, s.x, s.dy, s.offsets, s.perm, k.dw, ws=k.ws)
    return dict(dx=k.dx, dw=k.dw)


# ------------------------------------------------------------------ work

def work(case):
    """Each input read once (of the weights those of the experts that a uniform choice reaches), each output written
    once; the operations of the definition."""
    c = SimpleNamespace(**case)
    size = 2 if c.dtype == "bf16" else 4
    if c.mode in ("join", "join_back"):
        gates = c.T * {"none": 0, "token": 1, "channel": c.d}[c.gate]
        if c.mode == "join":  # in: x, y, gate, three vectors; out: x', n
            return {"bytes": c.T * c.d * (4 + 3 * size) + gates * size + 12 * c.d, "flops": 12.0 * c.T * c.d}
        # in: x', dx', dn, y, gate, three vectors; out: dx, dy, dgate, three vectors
        return {"bytes": c.T * c.d * (8 + 4 * size) + 2 * gates * size + 24 * c.d, "flops": 25.0 * c.T * c.d}
    N, M = c.rows * c.cols, c.T * c.K
    reached = N * (1 - (1 - c.K / N) ** c.T)
    matrix = (2 if case.get("swiglu") else 1) * c.n_out * c.n_in
    x, y = (c.T if c.x_order == "token" else M) * c.n_in * size, M * c.n_out * size
    index = 4 * (N + 1) + (0 if c.x_order == c.y_order == "position" else 4 * M)
    if c.mode == "product_back":  # in: x, dy, w; out: dx, dw (zeros where an expert has no rows)
        return {"bytes": x + y + M * c.n_in * size + (reached + N) * matrix * size + 4 * (N + 1) + 4 * M,
                "flops": 4.0 * M * matrix}
    weight = 17 / 32 if c.mode == "product4" else size
    return {"bytes": x + y + reached * matrix * weight + index, "flops": 2.0 * M * matrix}


# ------------------------------------------------------------------ the same in 64 bits

def _exact_join(case, seed):
    t = SimpleNamespace(**_join_tensors(case, seed))
    f64 = torch.float64
    x, y = t.x.to(f64), t.y.to(f64)
    w_out, w_in, a = t.w_out.to(f64), t.w_in.to(f64), t.scale.to(f64)
    d = x.shape[1]
    p = 1.0 if t.gate is None else 1 / (1 + torch.exp(-t.gate.to(f64)))
    sy = torch.sqrt(torch.linalg.vecdot(y, y)[:, None] / d + EPS)
    if case["mode"] == "join":
        z = x + a * p * w_out * y / sy
        return dict(x_out=z, n=w_in * z / torch.sqrt(torch.linalg.vecdot(z, z)[:, None] / d + EPS))
    dn = t.dn.to(f64)
    sx = torch.sqrt(torch.linalg.vecdot(x, x)[:, None] / d + EPS)
    # d(x / sx) = dx / sx - x <x, dx> / (d sx^3)
    v = dn * w_in
    G = t.dx_out.to(f64) + v / sx - x * torch.linalg.vecdot(x, v)[:, None] / (d * sx ** 3)
    k = G * p * a * w_out
    out = dict(dx=G, dy=k / sy - y * torch.linalg.vecdot(y, k)[:, None] / (d * sy ** 3), dw_in=(dn * x / sx).sum(0),
               dw_out=(G * p * a * y / sy).sum(0), dscale=(G * p * w_out * y / sy).sum(0))
    if t.gate is not None:
        dg = G * a * w_out * y / sy * p * (1 - p)
        out["dgate"] = dg.sum(1, keepdim=True) if case["gate"] == "token" else dg
    return out


def exact(case, seed):
    if case["mode"] in ("join", "join_back"):
        return _exact_join(case, seed)
    t = SimpleNamespace(**_product_tensors(case, seed))
    c, f64 = case, torch.float64
    K, M, n = c["K"], c["T"] * c["K"], c["n_out"]
    ends = t.offsets.tolist()
    at = {"position": torch.arange(M, device="cuda"), "task": t.perm.long(), "token": t.perm.long() // K}
    back = c["mode"] == "product_back"
    y = torch.zeros((M, c["n_in"] if back else n), dtype=f64, device="cuda")
    dw = torch.zeros((len(ends) - 1, n, c["n_in"]), dtype=f64, device="cuda") if back else None
    for e, (lo, hi) in enumerate(zip(ends[:-1], ends[1:])):
        if lo == hi:
            continue
        if c["mode"] == "product4":
            codes, k = t.codes[e].long(), c["n_in"]
            w = torch.empty((codes.shape[0], k), dtype=f64, device="cuda")
            for half in (0, 1):
                q = (codes >> (4 * half)) & 15
                ex, m = (q >> 1) & 3, (q & 1).to(f64)
                mag = torch.where(ex > 0, torch.ldexp(1 + m / 2, ex.to(f64) - 1), m / 2)
                w[:, half::2] = torch.where(q >= 8, -mag, mag)
            w *= torch.exp2(t.scales[e].to(f64) - 127).repeat_interleave(32, 1)
        else:
            w = t.w[e].to(f64)
        x = t.x[at[c["x_order"]][lo:hi]].to(f64)
        if back:
            dy = t.dy[at[c["y_order"]][lo:hi]].to(f64)
            y[at[_dx_order(c)][lo:hi]] = dy @ w
            dw[e] = dy.t() @ x
        elif c["swiglu"]:
            g = x @ w[:n].t()
            y[at[c["y_order"]][lo:hi]] = g / (1 + torch.exp(-g)) * (x @ w[n:].t())
        else:
            y[at[c["y_order"]][lo:hi]] = x @ w.t()
    return dict(dx=y, dw=dw) if back else dict(y=y)
