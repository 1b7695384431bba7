"""What is measured of the operators around the routed layer: the 8-bit activation checkpoint, the shared branch's way
back from it, the shared branch with the low-rank adapters of many requests, and the whole feed-forward layer for a few
tokens.

A case is a dict of plain values. Its ``mode`` is the call that a program makes:

* ``checkpoint``  omnimoe_checkpoint_store and omnimoe_checkpoint_load: an activation goes to 8 bits and comes back;
* ``backward``    omnimoe_shared_mlp_backward: gradients of the shared SwiGLU branch from the checkpoint of its input;
* ``adapters``    omnimoe_shared_mlp_adapters: the shared branch of a batch whose tokens belong to requests with
                  adapters of their own (or with none), added to the routed branch's output and
                  rounded to the layer's type;
* ``few``         omnimoe_layer_forward_few: Eq. 7 whole (routed and shared branch) for a decode step of a few tokens.

``listed()`` names the cases, ``draw(rng)`` gives others of the same ranges, ``prepare`` makes what the program holds
before the call, ``run`` makes the call (or, where ``own`` is false, computes the same in plain torch) and ``exact``
recomputes the outputs in 64 bits.
"""
from __future__ import annotations

import math
from types import SimpleNamespace

import torch

own = False

# The 1024 x 1024-expert layer of the training and decode workloads, the 256 x 256-expert one of the small workload,
# the 320 x 320 one of the paper's speed benchmark.
BIG = dict(d=2048, n_rows=1024, n_cols=1024, d_key=1024, H=8, K=16)
SMALL = dict(d=512, n_rows=256, n_cols=256, d_key=256, H=4, K=16)
PAPER = dict(d=1024, n_rows=320, n_cols=320, d_key=512, H=1, K=64)


def listed():
    return [
        # The input of a layer for a chunk of a batch, of a length that no tile divides; and the training batch's.
        dict(name="checkpoint_chunk", mode="checkpoint", T=509, d=2048, dtype="bf16"),
        dict(name="checkpoint_train", mode="checkpoint", T=16384, d=2048, dtype="bf16"),
        # The shared branch's way back: a small model's ragged batch, the fp32 layer of accuracy work, the training batch.
        dict(name="backward_small", mode="backward", T=4093, d=512, d_ff=512, dtype="bf16"),
        dict(name="backward_f32", mode="backward", T=1000, d=520, d_ff=520, dtype="f32"),
        dict(name="backward_train", mode="backward", T=16384, d=2048, d_ff=2048, dtype="bf16"),
        # One token of one request; a decode step of 64 requests with adapters of their own; the prompts of several
        # requests at once; a ragged batch in fp32 in which a third of the tokens have no adapter.
        dict(name="adapters_decode1", mode="adapters", T=1, d=2048, d_ff=2048, n=64, r=16, ids="own", dtype="bf16"),
        dict(name="adapters_decode64", mode="adapters", T=64, d=2048, d_ff=2048, n=64, r=16, ids="own", dtype="bf16"),
        dict(name="adapters_prefill", mode="adapters", T=4096, d=2048, d_ff=2048, n=16, r=32, ids="runs", dtype="bf16"),
        dict(name="adapters_f32", mode="adapters", T=333, d=520, d_ff=520, n=12, r=8, ids="mixed", dtype="f32"),
        # One decoded token and a decode step of sixteen on the training tables; seven tokens of a small fp32 layer.
        dict(BIG, name="few_decode1", mode="few", T=1, d_ff=2048, dtype="bf16", act="gelu", query="split"),
        dict(BIG, name="few_decode16", mode="few", T=16, d_ff=2048, dtype="bf16", act="gelu", query="split"),
        dict(SMALL, name="few_small_f32", mode="few", T=7, d_ff=512, dtype="f32", act="silu", query="split"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any of the modes, one token to the training batch, odd lengths and widths (multiples of 8, as the
    layer asks for) among them."""
    mode = rng.choice(["checkpoint", "backward", "adapters", "adapters", "few", "few"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if mode == "checkpoint":
        d = rng.choice([8 * _log_int(rng, 1, 512), 512, 1024, 2048, 4096])
        return dict(mode=mode, T=_log_int(rng, 1, min(32768, (1 << 25) // d)), d=d, dtype=dtype)
    if mode == "backward":
        d = rng.choice([8 * _log_int(rng, 8, 256), 512, 1024, 2048])
        d_ff = rng.choice([d, 8 * _log_int(rng, 8, 256), 2 * d])
        most = int((1 << 36) / (d * d_ff)) if dtype == "bf16" else int((1 << 31) / (d * d_ff))
        return dict(mode=mode, T=_log_int(rng, 16, max(64, min(16384, most))), d=d, d_ff=d_ff, dtype=dtype)
    if mode == "adapters":
        d = rng.choice([8 * _log_int(rng, 8, 256), 512, 1024, 2048])
        d_ff = rng.choice([d, 8 * _log_int(rng, 8, 512)])
        if dtype == "f32":
            d, d_ff = min(d, 1024), min(d_ff, 1024)
        T = _log_int(rng, 1, 4096 if dtype == "bf16" else 1024)
        return dict(mode=mode, T=T, d=d, d_ff=d_ff, n=_log_int(rng, 1, 128), r=rng.choice([8, 16, 16, 32, 64]),
                    ids=rng.choice(["own", "runs", "mixed"]), dtype=dtype)
    kind = rng.choice(["big", "small", "small", "paper"])
    act, query = rng.choice(["gelu", "gelu", "silu"]), "split"
    if kind == "big":
        tables, dtype, d_ff = dict(BIG), "bf16", 2048
    elif kind == "paper":
        tables, d_ff = dict(PAPER, K=rng.randint(1, 64)), 1024
    else:
        d = rng.choice([8 * rng.randint(8, 96), 512, 1024])
        query = rng.choice(["split", "split", "shared"])
        rows = rng.choice([rng.randint(16, 400), 64, 256, 512])
        tables = dict(d=d, n_rows=rows, n_cols=rows if rng.random() < 0.6 else rng.randint(16, 400),
                      d_key=d // 2 // 8 * 8 if query == "split" else d, H=rng.randint(1, 8),
                      K=rng.choice([1, 4, 8, 13, 16, 16, 32]))
        d_ff = rng.choice([0, d, 8 * rng.randint(1, 128)])
    return dict(tables, mode=mode, T=rng.randint(1, 16), d_ff=d_ff, dtype=dtype, act=act, query=query)


# ------------------------------------------------------------------ inputs

def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 32 + stream)
    return g


def _normal(case, seed, stream, shape, scale=1.0, dtype=None):
    dt = dtype or (torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)
    t = torch.randn(shape, generator=_gen(seed, stream), device="cuda", dtype=dt)
    return t.mul_(scale) if scale != 1.0 else t


def _steps(case, seed, stream, shape, scale, step):
    """N(0, scale^2) in whole multiples of ``step``, at most 256 of them, which both types hold."""
    t = torch.randn(shape, generator=_gen(seed, stream), device="cuda").mul_(scale / step).round_().clamp_(-256, 256)
    return t.mul_(step).to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32)


def _tensors(case, seed):
    """Activations ~ N(0, 1), weights ~ N(0, 1 / their inner width)."""
    c = SimpleNamespace(**case)
    T, d = c.T, c.d
    w = 1.0 / math.sqrt(d)
    if c.mode == "checkpoint":
        x = _normal(case, seed, 1, (T, d))
        # channels of very different size, as a residual stream has them
        return dict(x=x.mul_(torch.exp2(2.0 * torch.randn((d,), generator=_gen(seed, 2), device="cuda")).to(x.dtype)))
    if c.mode == "backward":
        codes, scales = _quantise(_normal(case, seed, 1, (T, d)).float())
        return dict(codes=codes.view(torch.uint8), scales=scales, w_gu=_normal(case, seed, 3, (2 * c.d_ff, d), w),
                    w_down=_normal(case, seed, 4, (d, c.d_ff), 1.0 / math.sqrt(c.d_ff)),
                    # the loss's gradient at the layer's output, averaged over the batch's tokens, and the routed
                    # branch's share of dL/dx, to which the call adds its own
                    dy=_normal(case, seed, 5, (T, d), 1.0 / T, torch.float32),
                    dx_in=_normal(case, seed, 6, (T, d), 1.0 / T, torch.float32))
    if c.mode == "adapters":
        if c.ids == "own":       # a token of each request: requests in any order, an adapter each
            ids = torch.randperm(max(c.T, c.n), generator=_gen(seed, 2), device="cuda")[:c.T] % c.n
        elif c.ids == "runs":    # prompts one after the other
            ids = torch.arange(c.T, device="cuda") * c.n // c.T
        else:                    # in any order, about a third without an adapter
            ids = torch.randint(-((c.n + 1) // 2), c.n, (c.T,), generator=_gen(seed, 2), device="cuda").clamp_(min=-1)
        return dict(ids=ids.to(torch.int32), x=_normal(case, seed, 1, (T, d)),
                    w_gu=_normal(case, seed, 3, (2 * c.d_ff, d), w),
                    w_down=_normal(case, seed, 4, (d, c.d_ff), 1.0 / math.sqrt(c.d_ff)),
                    a_gu=_normal(case, seed, 5, (c.n, 2 * c.r, d), w),
                    b_gu=_normal(case, seed, 6, (c.n, 2 * c.d_ff, c.r), 0.5 / math.sqrt(c.r)),
                    a_down=_normal(case, seed, 7, (c.n, c.r, c.d_ff), 1.0 / math.sqrt(c.d_ff)),
                    b_down=_normal(case, seed, 8, (c.n, d, c.r), 0.5 / math.sqrt(c.r)),
                    scale=torch.rand((c.n,), generator=_gen(seed, 9), device="cuda") + 0.5,
                    y_in=_normal(case, seed, 10, (T, d), 1.0, torch.float32))
    # Token values in sixteenths and sub-key values in 1/1024ths: every sum of their products is exact in 32 bits, so
    # that the logits, and with them the choice of the experts, are the same in any order of the sums; equal scores
    # come up, and go to the lower id.
    N = c.n_rows * c.n_cols
    t = dict(x=_steps(case, seed, 1, (T, d), 1.0, 1 / 16),
             keys_row=_steps(case, seed, 2, (c.H, c.n_rows, c.d_key), w, 1 / 1024),
             keys_col=_steps(case, seed, 3, (c.H, c.n_cols, c.d_key), w, 1 / 1024),
             u=_normal(case, seed, 4, (N, d), w), v=_normal(case, seed, 5, (N, d), w), w_gu=None, w_down=None)
    if c.d_ff:
        t["w_gu"] = _normal(case, seed, 6, (2 * c.d_ff, d), w)
        t["w_down"] = _normal(case, seed, 7, (d, c.d_ff), 1.0 / math.sqrt(c.d_ff))
    return t


def prepare(case, seed):
    return SimpleNamespace(case=dict(case), kept=None, **_tensors(case, seed))


# ------------------------------------------------------------------ the plain forms

def _quantise(x):
    """(e4m3 codes, scale bytes) of the rows' blocks of 32: the scale is the least power of two, 2^-127 at least, that
    brings the block's largest magnitude to 448 or below; its byte is the exponent plus 127."""
    T, d = x.shape
    blocks = -(-d // 32)
    b = torch.nn.functional.pad(x, (0, blocks * 32 - d)).view(T, blocks, 32)
    m, e = torch.frexp(b.abs().amax(-1))
    s = torch.where(m > 0, e - 9 + (m > 0.875), -127).clamp_(min=-127)
    q = (b.double() * torch.exp2(-s.double()).unsqueeze(-1)).float().to(torch.float8_e4m3fn)
    return q.view(T, blocks * 32)[:, :d].contiguous(), (s + 127).to(torch.uint8)


def _dequantise(codes, scales):
    T, d = codes.shape
    s = torch.exp2(scales.double() - 127).repeat_interleave(32, 1)[:, :d]
    return (codes.float().double() * s).float()


def _plain_backward(s):
    x = _dequantise(s.codes.view(torch.float8_e4m3fn), s.scales)
    w_gu, w_down = s.w_gu.float(), s.w_down.float()
    g, u = (x @ w_gu.t()).chunk(2, 1)
    sg = torch.sigmoid(g)
    da = s.dy @ w_down
    dh = torch.cat((da * u * (sg * (1 + g * (1 - sg))), da * g * sg), 1)
    dt = s.w_gu.dtype
    return dict(dx=(s.dx_in + dh @ w_gu).to(dt), dw_gu=(dh.t() @ x).to(dt), dw_down=(s.dy.t() @ (g * sg * u)).to(dt))


def _plain_adapters(s):
    r = s.b_gu.shape[2]
    ids = s.ids.long().clamp(min=0)
    scale = torch.where(s.ids >= 0, s.scale[ids], 0.0)[:, None]
    x = s.x.float()
    low = scale * (s.a_gu[ids].float() @ x[:, :, None])[:, :, 0]
    b_gate, b_up = s.b_gu[ids].float().chunk(2, 1)
    g, u = (x @ s.w_gu.float().t()).chunk(2, 1)
    g = g + (b_gate @ low[:, :r, None])[:, :, 0]
    u = u + (b_up @ low[:, r:, None])[:, :, 0]
    a = g * torch.sigmoid(g) * u
    low = scale * (s.a_down[ids].float() @ a[:, :, None])[:, :, 0]
    y = s.y_in + (a @ s.w_down.float().t() + (s.b_down[ids].float() @ low[:, :, None])[:, :, 0])
    return dict(y=y.to(s.x.dtype))


def _best_cells(c, row, col, K):
    """The K best cells of each grid row[i] + col[j] by (score descending, id ascending): ids and scores in 64 bits.
    They lie among the K best rows and the K best columns."""
    r, ri = torch.sort(row.double(), dim=-1, descending=True, stable=True)
    q, qi = torch.sort(col.double(), dim=-1, descending=True, stable=True)
    r, ri, q, qi = r[..., :K], ri[..., :K], q[..., :K], qi[..., :K]
    score = (r.unsqueeze(-1) + q.unsqueeze(-2)).flatten(-2)
    ids = (ri.unsqueeze(-1) * c["n_cols"] + qi.unsqueeze(-2)).flatten(-2)
    ids, at = torch.sort(ids, dim=-1)
    score, best = torch.sort(torch.gather(score, -1, at), dim=-1, descending=True, stable=True)
    return torch.gather(ids, -1, best)[..., :K], score[..., :K]


def _plain_few(s):
    c = s.case
    T, H, K, dk = c["T"], c["H"], c["K"], c["d_key"]
    x = s.x.float()
    c0 = dk if c["query"] == "split" else 0
    row = (x[:, :dk] @ s.keys_row.float().flatten(0, 1).t()).view(T, H, -1)
    col = (x[:, c0:c0 + dk] @ s.keys_col.float().flatten(0, 1).t()).view(T, H, -1)
    idx, score = _best_cells(c, row, col, K)
    e = torch.exp((score - score[..., :1]).float())
    gates = e / e.sum(-1, keepdim=True)
    at = idx.flatten(1)
    h = (s.u[at].float() @ x[:, :, None])[:, :, 0]
    act = h * torch.sigmoid(h) if c["act"] == "silu" else 0.5 * h * torch.erfc(h * -math.sqrt(0.5))
    y = ((gates.flatten(1) * act)[:, None] @ s.v[at].float())[:, 0]
    if c["d_ff"]:
        g, u = (x @ s.w_gu.float().t()).chunk(2, 1)
        y = y + (g * torch.sigmoid(g) * u) @ s.w_down.float().t()
    return dict(y=y, idx=idx.to(torch.int32), gates=gates)


# ------------------------------------------------------------------ the framework's calls

def _kept(s):
    """Descriptor, outputs and workspace, made at the first pass and kept, as a program does."""
    import paper_2602_05711_amd as P
    c = s.case
    layer = {k: c.get(k, v) for k, v in SMALL.items()}
    if c["mode"] != "few":
        layer["d_key"] = 8
    if c["mode"] == "checkpoint" and c["d"] < 16:
        layer["query_mode"] = "shared"
    desc = P.make_desc(SimpleNamespace(T=c["T"], dtype=c["dtype"], act=c.get("act", "gelu"), group_size=1,
                                       query_mode=layer.pop("query_mode", c.get("query", "split")), **layer))
    k = SimpleNamespace(P=P, desc=desc)
    T, d = c["T"], c["d"]

    def new(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda")

    def workspace(n):
        return new((max(n, 256),), torch.uint8)

    if c["mode"] == "checkpoint":
        k.codes, k.scales = new((T, d), torch.uint8), new((T, -(-d // 32)), torch.uint8)
        k.back = torch.empty_like(s.x)
    elif c["mode"] == "backward":
        k.dx, k.dw_gu, k.dw_down = new((T, d), s.w_gu.dtype), torch.empty_like(s.w_gu), torch.empty_like(s.w_down)
        k.ws = workspace(P.omnimoe_shared_mlp_backward_workspace_size(desc, c["d_ff"]))
    elif c["mode"] == "adapters":
        k.adapters = P.make_adapters(s.a_gu, s.b_gu, s.a_down, s.b_down, s.scale)
        k.y = torch.empty_like(s.x)
        k.ws = workspace(P.omnimoe_shared_mlp_adapters_workspace_size(desc, c["d_ff"], k.adapters))
    else:
        k.y = new((T, d), torch.float32)
        k.idx, k.gates = new((T, c["H"], c["K"]), torch.int32), new((T, c["H"], c["K"]), torch.float32)
        k.ws = workspace(P.omnimoe_layer_few_workspace_size(desc, c["d_ff"]))
    return k


def run(s):
    mode = s.case["mode"]
    if not own:
        if mode == "checkpoint":
            codes, scales = _quantise(s.x.float())
            return dict(x=_dequantise(codes, scales).to(s.x.dtype), scales=scales)
        return {"backward": _plain_backward, "adapters": _plain_adapters, "few": _plain_few}[mode](s)
    if s.kept is None:
        s.kept = _kept(s)
    k = s.kept
    if mode == "checkpoint":
        k.P.omnimoe_checkpoint_store(k.desc, s.x, k.codes, k.scales)
        k.P.omnimoe_checkpoint_load(k.desc, k.codes, k.scales, k.back)
        return dict(x=k.back, scales=k.scales)
    if mode == "backward":
        k.P.omnimoe_shared_mlp_backward(k.desc, s.case["d_ff"], s.codes, s.scales, s.w_gu, s.w_down, s.dy, s.dx_in,
                                        k.dx, k.dw_gu, k.dw_down, ws=k.ws)
        return dict(dx=k.dx, dw_gu=k.dw_gu, dw_down=k.dw_down)
    if mode == "adapters":
        k.P.omnimoe_shared_mlp_adapters(k.desc, s.case["d_ff"], k.adapters, s.x, s.w_gu, s.w_down, s.ids, s.y_in, k.y,
                                        ws=k.ws)
        return dict(y=k.y)
    k.P.omnimoe_layer_forward_few(k.desc, s.case["d_ff"], s.x, s.keys_row, s.keys_col, s.u, s.v, s.w_gu, s.w_down, k.y,
                                  k.idx, k.gates, ws=k.ws)
    return dict(y=k.y, idx=k.idx, gates=k.gates)


# ------------------------------------------------------------------ work

def work(case):
    """Each input read once (of the expert tables and the adapters the rows that the tokens reach at least: of "own"
    and "mixed" ids as many adapters as a uniform choice reaches), each output written once; the products of the
    definition, the recomputed projections of the way back among them."""
    c = SimpleNamespace(**case)
    size = 2 if c.dtype == "bf16" else 4
    if c.mode == "checkpoint":  # in: x; out: codes and scales; in: both; out: x
        return {"bytes": c.T * c.d * (2 * size + 2) + 2 * c.T * -(-c.d // 32), "flops": 2.0 * c.T * c.d}
    x, mlp = c.T * c.d, 3 * c.d * c.d_ff
    if c.mode == "backward":
        # in: codes, scales, weights, dy, dx_in; out: dx, weight gradients
        return {"bytes": x + c.T * -(-c.d // 32) + 2 * mlp * size + (8 + size) * x,
                "flops": 16.0 * c.T * c.d * c.d_ff}
    if c.mode == "adapters":
        with_one = c.T * (2 / 3 if c.ids == "mixed" else 1)
        reached = min(c.n, c.T) if c.ids != "mixed" else c.n * -math.expm1(-with_one / c.n)
        per_token = 2 * c.r * c.d + 2 * c.r * c.d_ff + c.r * c.d_ff + c.r * c.d
        return {"bytes": x * (2 * size + 4) + mlp * size + reached * per_token * size + 4 * c.T + 4 * reached,
                "flops": 2.0 * c.T * mlp + 2.0 * with_one * per_token}
    M, N = c.T * c.H * c.K, c.n_rows * c.n_cols
    keys = c.H * (c.n_rows + c.n_cols) * c.d_key
    return {"bytes": x * (size + 4) + (keys + mlp) * size + 2 * N * -math.expm1(-M / N) * c.d * size + 8 * M,
            "flops": 2.0 * c.T * (keys + mlp) + 4.0 * M * c.d}


# ------------------------------------------------------------------ the same in 64 bits

def _exact_checkpoint(x):
    """Rounds to e4m3 by its definition: three bits after the leading one, exponents from -6 on, the even neighbour
    where two are as near."""
    T, d = x.shape
    b = torch.zeros((T, -(-d // 32) * 32), dtype=torch.float64, device=x.device)
    b[:, :d] = x
    b = b.view(T, -1, 32)
    most = b.abs().amax(-1, keepdim=True)
    s = torch.ceil(torch.log2(torch.where(most > 0, most, 1.0) / 448.0))
    s = s + (most > 448.0 * torch.exp2(s)).double() - (most <= 448.0 * torch.exp2(s - 1)).double()
    s = torch.where(most > 0, s, -127.0).clamp(min=-127.0)
    v = b / torch.exp2(s)
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(v / step) * step * torch.exp2(s)).view(T, -1)[:, :d]


def exact(case, seed):
    t = SimpleNamespace(**_tensors(case, seed))
    f64 = torch.float64
    if case["mode"] == "checkpoint":
        return dict(x=_exact_checkpoint(t.x.to(f64)), scales=None)
    T, d, f = case["T"], case["d"], case["d_ff"]
    if case["mode"] == "backward":
        byte = t.codes.long()
        e, m = (byte >> 3) & 15, (byte & 7).to(f64)
        mag = torch.where(e > 0, torch.ldexp(8 + m, e.to(f64) - 10), torch.ldexp(m, torch.full_like(m, -9.0)))
        block = torch.arange(d, device="cuda") // 32
        x = torch.where(byte > 127, -mag, mag) * torch.exp2(t.scales.to(f64)[:, block] - 127)
        gu, dn, dy = t.w_gu.to(f64), t.w_down.to(f64), t.dy.to(f64)
        gate, up = x @ gu[:f].t(), x @ gu[f:].t()
        p = 1 / (1 + torch.exp(-gate))
        da = dy @ dn
        dg, du = da * up * p * (1 + gate * (1 - p)), da * gate * p
        return dict(dx=t.dx_in.to(f64) + dg @ gu[:f] + du @ gu[f:], dw_gu=torch.cat((dg.t() @ x, du.t() @ x)),
                    dw_down=dy.t() @ (gate * p * up))
    x = t.x.to(f64)
    if case["mode"] == "adapters":
        gu, y = x @ t.w_gu.to(f64).t(), t.y_in.to(f64)
        rows = [(i, (t.ids == i).nonzero().flatten()) for i in range(case["n"])]
        r = case["r"]
        for i, at in rows:
            if at.numel():
                low = float(t.scale[i]) * (x[at] @ t.a_gu[i].to(f64).t())
                b = t.b_gu[i].to(f64)
                gu[at] += torch.cat((low[:, :r] @ b[:f].t(), low[:, r:] @ b[f:].t()), 1)
        a = gu[:, :f] / (1 + torch.exp(-gu[:, :f])) * gu[:, f:]
        y += a @ t.w_down.to(f64).t()
        for i, at in rows:
            if at.numel():
                y[at] += float(t.scale[i]) * (a[at] @ t.a_down[i].to(f64).t()) @ t.b_down[i].to(f64).t()
        return dict(y=y)
    H, K, nr, nc, dk = case["H"], case["K"], case["n_rows"], case["n_cols"], case["d_key"]
    xr, xc = x[:, :dk], x[:, dk:2 * dk] if case["query"] == "split" else x[:, :dk]
    y = torch.zeros((T, d), dtype=f64, device="cuda")
    gates = torch.empty((T, H, K), dtype=f64, device="cuda")
    for h in range(H):
        sr, sc = xr @ t.keys_row[h].to(f64).t(), xc @ t.keys_col[h].to(f64).t()
        for tok in range(T):
            grid = (sr[tok][:, None] + sc[tok]).flatten()
            least = torch.topk(grid, K).values[-1]
            ids = (grid >= least).nonzero().flatten()  # ascending, so that the stable sort keeps the lower id first
            order = torch.sort(grid[ids], descending=True, stable=True).indices[:K]
            ids = ids[order]
            gates[tok, h] = torch.softmax(grid[ids], 0)
            z = t.u[ids].to(f64) @ x[tok]
            z = z / (1 + torch.exp(-z)) if case["act"] == "silu" else 0.5 * z * (1 + torch.erf(z / math.sqrt(2.0)))
            y[tok] += (gates[tok, h] * z) @ t.v[ids].to(f64)
    if f:
        gate, up = x @ t.w_gu[:f].to(f64).t(), x @ t.w_gu[f:].to(f64).t()
        y += (gate / (1 + torch.exp(-gate)) * up) @ t.w_down.to(f64).t()
    return dict(y=y, idx=None, gates=gates)
