"""The operators of include/omnimoe_block.h on the GPU against plain 64-bit forms, within bounds derived from their
roundings (block_support), at the sizes, orders and values where they could go wrong; their use under graph capture, on
other streams and side by side; and a training and a decode step in which they run with the router and the schedule."""
from types import SimpleNamespace

import pytest

import synth  # noqa: F401  (the package's root on the path)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import block_support as K  # noqa: E402
import ffn_support as S  # noqa: E402
import paper_2602_05711_amd as P  # noqa: E402
from test_gpu_ffn_ops import BF16, F32, F64, TYPES, Guarded, tid, within  # noqa: E402

INF, NAN = float("inf"), float("nan")


def same_bits(a, b):
    kind = {2: torch.int16, 4: torch.int32}[a.element_size()]
    return torch.equal(a.view(kind), b.view(kind))


# ------------------------------------------------------------------ the joint

def _join_inputs(T, d, dtype, gate="channel", absent=(), seed=0):
    wide = torch.exp2(S.randn(seed + 9, 1, d, scale=1.5))
    i = SimpleNamespace(T=T, d=d, dtype=dtype, D=S.desc(T, d, dtype), eps=1e-5, x=(S.randn(seed, T, d) * wide).to(dtype),
                        y=S.randn(seed + 1, T, d, scale=0.3),
                        gate=S.randn(seed + 2, T, 1 if gate == "token" else d, scale=2.0, dtype=dtype),
                        w_out=S.randn(seed + 3, d) * 0.2 + 1, scale=S.randn(seed + 4, d) * 0.1 + 0.5,
                        w_in=S.randn(seed + 5, d) * 0.2 + 1, dx_out=S.randn(seed + 6, T, d, dtype=dtype),
                        dn=S.randn(seed + 7, T, d, dtype=dtype))
    if gate == "none":
        i.gate = None
    for k in absent:
        setattr(i, k, None)
    if i.y is None:
        i.gate = i.w_out = i.scale = None
    return i


def _wide(i, *names):
    return [None if getattr(i, n) is None else getattr(i, n).to(F64) for n in names]


def _join(i, stream=None):
    x_out, n = Guarded((i.T, i.d), i.dtype), Guarded((i.T, i.d), i.dtype)
    P.omnimoe_block_join(i.D, i.eps, i.x, i.y, i.gate, i.w_out, i.scale, i.w_in, None if i.y is None else x_out.t,
                         None if i.w_in is None else n.t, stream=stream)
    torch.cuda.synchronize()
    x_out.check()
    n.check()
    return i.x if i.y is None else x_out.t, None if i.w_in is None else n.t


def _join_back(i, x_out, stream=None, dx=None):
    new = lambda shape, dtype, there: Guarded(shape, dtype) if there else None  # noqa: E731
    T, d, v = i.T, i.d, (i.d,)
    o = dict(dx=Guarded((T, d), i.dtype), dy=new((T, d), F32, i.y is not None),
             dgate=None if i.gate is None else Guarded(tuple(i.gate.shape), i.dtype),
             dw_out=new(v, F32, i.w_out is not None), dscale=new(v, F32, i.scale is not None),
             dw_in=new(v, F32, i.w_in is not None))
    ws = Guarded((P.omnimoe_block_join_backward_workspace_size(i.D),), torch.uint8)
    ws.t.fill_(0xFF)
    t = {k: None if g is None else g.t for k, g in o.items()}
    if dx is not None:
        t["dx"] = dx
    P.omnimoe_block_join_backward(i.D, i.eps, x_out, i.y, i.gate, i.w_out, i.scale, i.w_in, i.dx_out, i.dn, t["dx"], t["dy"],
                                  t["dgate"], t["dw_out"], t["dscale"], t["dw_in"], ws=ws.t, stream=stream)
    torch.cuda.synchronize()
    for g in (*o.values(), ws):
        if g is not None:
            g.check()
    return {k: g for k, g in t.items() if g is not None}


SHAPES = [(1, 8), (1, 2048), (3, 520), (65, 1000), (7, 4096), (2500, 64), (5000, 512), (301, 2048)]
ABSENT = [(), ("w_out",), ("scale",), ("w_in",), ("y",), ("w_out", "scale"), ("w_out", "scale", "w_in")]


def _check_join(i, what):
    x_out, n = _join(i)
    (z, m), (bz, bn) = K.join_bounds(*_wide(i, "x", "y", "gate", "w_out", "scale", "w_in"), i.eps, i.dtype)
    within(x_out, z, bz, f"{what} x_out")
    if n is not None:
        within(n, m, bn, f"{what} n")
    return x_out


def _check_back(i, x_out, what):
    got = _join_back(i, x_out)
    args = [x_out.to(F64)] + _wide(i, "y", "gate", "w_out", "scale", "w_in", "dx_out", "dn")
    want, bound = K.join_back_bounds(*args, i.eps, i.dtype)
    assert sorted(got) == sorted(want)
    for k in want:
        within(got[k], want[k], bound[k], f"{what} {k}")


@pytest.mark.parametrize("gate", ["none", "token", "channel"])
@pytest.mark.parametrize("dtype", TYPES, ids=tid)
@pytest.mark.parametrize("T,d", SHAPES + [(4, 8192)])
def test_join_both_ways(T, d, dtype, gate):
    if dtype is F32 and d > 4096:
        d = 4088
    i = _join_inputs(T, d, dtype, gate)
    _check_back(i, _check_join(i, "join"), "join")


@pytest.mark.parametrize("absent", ABSENT, ids="-".join)
@pytest.mark.parametrize("gate", ["none", "channel"])
@pytest.mark.parametrize("dtype", TYPES, ids=tid)
def test_join_without(dtype, gate, absent):
    i = _join_inputs(37, 264, dtype, gate, absent, seed=20)
    x_out = _check_join(i, "join")
    _check_back(i, x_out, "join")
    if i.w_in is not None:
        i.dx_out = None
        _check_back(i, x_out, "no dx_out")


@pytest.mark.parametrize("dtype", TYPES, ids=tid)
def test_join_gates_at_their_ends(dtype):
    # sigmoid and its complement keep their relative accuracy; an infinite gate is a factor of 0 or 1
    i = _join_inputs(64, 72, dtype, "channel", seed=30)
    i.gate = torch.linspace(-80, 80, 64 * 72).view(64, 72).to(dtype).cuda()
    _check_back(i, _check_join(i, "gates"), "gates")
    i.gate[5, 7], i.gate[6, 8] = INF, -INF
    x_out = _check_join(i, "infinite gates")
    got = _join_back(i, x_out)
    assert float(x_out[6, 8]) == float(i.x[6, 8])
    assert float(got["dgate"][5, 7]) == 0 and float(got["dgate"][6, 8]) == 0 and all(bool(torch.isfinite(v).all()) for v in got.values())


@pytest.mark.parametrize("dtype", TYPES, ids=tid)
def test_join_extreme_rows(dtype):
    # rows of zeros, rows near the type's largest value, and rows whose squares are below fp32's range
    i = _join_inputs(6, 136, dtype, "token", seed=40)
    big = 2.0 ** 126
    i.y[1] = 0
    i.y[2] = torch.sign(i.y[2]) * big * (1 + torch.rand(136, device="cuda"))
    i.y[3] *= 2.0 ** -100
    i.x[4] = 0
    i.x[5] = (torch.sign(i.x[5].float()) * big * (1 + 0.5 * torch.rand(136, device="cuda"))).to(dtype)
    i.eps = 1e-30
    x_out = _check_join(i, "extreme")
    i.dx_out = torch.zeros_like(i.dx_out)
    _check_back(i, x_out, "extreme")


@pytest.mark.parametrize("gate", ["none", "token", "channel"])
@pytest.mark.parametrize("d,dtype", [(8192, BF16), (5000, BF16), (4096, F32), (1024, BF16), (512, F32)])
def test_join_of_the_largest_values(d, dtype, gate):
    # whole rows of the types' largest values: the sum of their squares, formed of smaller units, is in range at every width
    i = _join_inputs(4, d, dtype, gate, seed=41)
    i.y[1] = torch.sign(i.y[1]) * torch.finfo(F32).max
    i.x[2] = torch.sign(i.x[2]) * torch.finfo(dtype).max
    i.y[3], i.x[3] = i.y[1], i.x[2] * 0.75
    i.gate = None if i.gate is None else i.gate.clamp(max=0)  # (the sum of x and the branch stays in range)
    x_out = _check_join(i, "largest")
    _check_back(i, x_out, "largest")


@pytest.mark.parametrize("d", [8, 520, 2048])
def test_join_of_small_values_beside_a_large_one(d):
    # the row's squares pass fp32's range; the norms of its other values, far below them, are still normal numbers (2^-125)
    i = _join_inputs(3, d, F32, "none", ("scale",), seed=42)
    some = lambda seed: torch.sign(S.randn(seed, 3, d)) * (1 + S.randn(seed + 1, 3, d).abs().clamp(max=1))  # noqa: E731
    i.w_out, i.w_in = i.w_out.clamp(0.75, 1.25), i.w_in.clamp(0.75, 1.25)
    i.x.zero_()
    i.y = some(43) * 2.0 ** -60
    i.y[:, 3] = 1.5 * 2.0 ** 64
    _check_join(i, "beside")
    i.x, i.dx_out, i.dn = some(45) * 2.0 ** -60, some(47), some(49)
    i.x[:, 3] = 1.5 * 2.0 ** 64
    _check_back(i, i.x, "beside")


@pytest.mark.parametrize("dtype", TYPES, ids=tid)
def test_join_with_the_largest_eps(dtype):
    # a finite mean square and eps whose sum is past fp32's largest value
    i = _join_inputs(5, 72, dtype, "channel", seed=45)
    i.eps = float(torch.finfo(F32).max)
    i.x *= 2.0 ** 59
    i.y *= 2.0 ** 61
    _check_back(i, _check_join(i, "eps"), "eps")


@pytest.mark.parametrize("bad", [INF, -INF, NAN])
@pytest.mark.parametrize("where", ["x", "y", "gate"])
def test_join_keeps_what_is_not_finite_in_its_row(where, bad):
    i = _join_inputs(9, 1032, BF16, "channel", seed=50)
    clean_x, clean_n = _join(i)
    clean = _join_back(i, clean_x)
    getattr(i, where)[4, 517] = bad
    x_out, n = _join(i)
    others = torch.arange(9, device="cuda") != 4
    assert same_bits(x_out[others], clean_x[others]) and same_bits(n[others], clean_n[others])
    got = _join_back(i, x_out)
    for k in ("dx", "dy", "dgate"):
        assert same_bits(got[k][others].contiguous(), clean[k][others].contiguous()), k
    if where == "y" or bad != bad:
        assert not bool(torch.isfinite(x_out[4]).all()) and not bool(torch.isfinite(got["dx"][4].float()).all())


@pytest.mark.parametrize("gate", ["none", "token", "channel"])
@pytest.mark.parametrize("dtype", TYPES, ids=tid)
@pytest.mark.parametrize("bad", [INF, NAN])
def test_join_without_its_norm_passes_gradients_by_y(bad, dtype, gate):
    # dy is the branch's factor times the stream's gradient, whatever y holds, with every form of the gate
    i = _join_inputs(5, 264, dtype, gate, ("w_out",), seed=55)
    x_out = i.x.clone()
    clean = _join_back(i, x_out)
    i.y[2, 100] = bad
    got = _join_back(i, x_out)
    assert same_bits(got["dy"], clean["dy"]) and bool(torch.isfinite(got["dy"]).all())
    assert same_bits(got["dx"], clean["dx"]) and same_bits(got["dw_in"], clean["dw_in"])


@pytest.mark.parametrize("dtype", TYPES, ids=tid)
def test_join_in_place(dtype):
    i = _join_inputs(33, 520, dtype, seed=60)
    x_out, n = _join(i)
    clean = _join_back(i, x_out)
    x, m = i.x.clone(), torch.empty_like(i.x)
    P.omnimoe_block_join(i.D, i.eps, x, i.y, i.gate, i.w_out, i.scale, i.w_in, x, m)
    assert same_bits(x, x_out) and same_bits(m, n)
    for name in ("dx_out", "dn"):
        kept = getattr(i, name)
        setattr(i, name, kept.clone())
        got = _join_back(i, x_out, dx=getattr(i, name))
        assert all(same_bits(got[k], clean[k]) for k in clean), name
        setattr(i, name, kept)


def test_join_of_no_tokens():
    i = _join_inputs(0, 64, BF16, "token")
    P.omnimoe_block_join(i.D, i.eps, None, None, None, None, None, i.w_in, None, None)
    got = _join_back(i, i.x)
    assert all(int(got[k].count_nonzero()) == 0 for k in ("dw_out", "dscale", "dw_in"))


def test_join_backward_of_no_tokens_with_one_output():
    # of the sums each may be asked for alone, and nothing else has to be there
    D = S.desc(0, 64, BF16)
    for k in ("dw_out", "dscale", "dw_in"):
        out = dict.fromkeys(("dw_out", "dscale", "dw_in"))
        out[k] = torch.full((64,), 3.0, device="cuda")
        P.omnimoe_block_join_backward(D, 1e-6, None, None, None, None, None, None, None, None, None, None, None, **out)
        assert int(out[k].count_nonzero()) == 0
    P.omnimoe_block_join_backward(D, 1e-6, *[None] * 14)


def test_join_of_a_long_batch():
    # rows past 2^31 values
    T, d = 300000, 8192
    D = S.desc(T, d, BF16)
    x = torch.zeros((T, d), dtype=BF16, device="cuda")
    x[-1], x[T // 2] = 3.0, -2.0
    n = torch.full_like(x, 7.0)
    w = torch.ones(d, device="cuda")
    P.omnimoe_block_join(D, 1e-6, x, None, None, None, None, w, None, n)
    assert bool((n[-1] == 1).all()) and bool((n[T // 2] == -1).all()) and int(n[:T // 2].count_nonzero()) == 0


# ------------------------------------------------------------------ products

ORDERS = [("position", "position"), ("token", "position"), ("task", "task"), ("position", "task"), ("token", "task")]


def _case(T, H, Kk, grid, n_in, n_out, dtype, swiglu=False, orders=("token", "position"), idx=None, seed=0,
          weights=True):
    N, M = grid[0] * grid[1], T * H * Kk
    g = torch.Generator().manual_seed(seed + 77)
    if idx is None:
        idx = (torch.rand(M, generator=g) ** 2 * N).long().clamp(max=N - 1)
    perm, offsets = K.schedule(torch.as_tensor(idx), N)
    c = SimpleNamespace(T=T, hk=H * Kk, N=N, M=M, k=n_in, n=n_out, dtype=dtype, swiglu=swiglu, orders=orders,
                        D=S.desc(T, 64, dtype, n_rows=grid[0], n_cols=grid[1], H=H, K=Kk, query_mode="shared"),
                        q=P.make_product(n_in, n_out, swiglu, *orders), perm=perm.cuda(), offsets=offsets.cuda(),
                        x=S.randn(seed, T if orders[0] == "token" else M, n_in, dtype=dtype),
                        w=None if not weights else S.randn(seed + 1, N, (2 if swiglu else 1) * n_out, n_in, scale=n_in ** -0.5,
                                                           dtype=dtype),
                        dy=S.randn(seed + 2, M, n_out, dtype=dtype))
    if N == 1 and M:
        c.offsets = None
    return c


def _ends(c):
    return torch.tensor([0, c.M], device="cuda") if c.offsets is None else c.offsets


def _by_position(c, t, order):
    return t[K.rows_of(c.perm, order, c.hk, c.M, "cuda")].to(F64)


def _written(c, got, order):
    """The rows of an output by position."""
    return got[K.rows_of(c.perm, order, c.hk, c.M, "cuda")]


def _perm(c, *orders):
    return None if all(o == "position" for o in orders) else c.perm


def _run(c, fn, *tensors, shape, orders, q=None):
    out = Guarded(shape, c.dtype)
    out.t.fill_(float("nan"))
    getattr(P, fn)(c.D, c.q if q is None else q, *tensors, c.offsets, _perm(c, *orders), out.t)
    torch.cuda.synchronize()
    out.check()
    return out.t


def _check_product(c, fn="omnimoe_grouped_product", weights=None, w=None):
    got = _run(c, fn, c.x, *(weights or (c.w,)), shape=(c.M, c.n), orders=c.orders)
    want, bound = K.product(_by_position(c, c.x, c.orders[0]), c.w if w is None else w, _ends(c), c.swiglu, c.dtype)
    within(_written(c, got, c.orders[1]), want, bound, fn)
    return got


def _check_product_back(c):
    x_order = "task" if c.orders[0] == "token" else c.orders[0]
    q = P.make_product(c.k, c.n, False, x_order, c.orders[1])
    dx = _run(c, "omnimoe_grouped_product_dx", c.dy, c.w, shape=(c.M, c.k), orders=(x_order, c.orders[1]), q=q)
    dy = _by_position(c, c.dy, c.orders[1])
    within(_written(c, dx, x_order), *K.product_dx(dy, c.w, _ends(c), c.dtype), "dx")
    return dx, _check_dw(c)


def _check_dw(c):
    dw = Guarded((c.N, c.n, c.k), c.dtype)
    dw.t.fill_(float("nan"))
    ws = Guarded((max(256, P.omnimoe_grouped_product_dw_workspace_size(c.D, c.q)),), torch.uint8)
    ws.t.fill_(0xFF)
    P.omnimoe_grouped_product_dw(c.D, c.q, c.x, c.dy, c.offsets, _perm(c, *c.orders), dw.t, ws=ws.t)
    torch.cuda.synchronize()
    dw.check()
    ws.check()
    dy = _by_position(c, c.dy, c.orders[1])
    within(dw.t, *K.product_dw(_by_position(c, c.x, c.orders[0]), dy, _ends(c), c.dtype), "dw")
    return dw.t


# one token, few rows, ragged tiles of every side, one expert (no offsets), many experts, heads
PRODUCTS = [(1, 1, 1, (1, 1), 8, 8), (1, 1, 8, (8, 8), 2048, 72), (16, 1, 8, (8, 8), 136, 264), (5, 2, 3, (2, 3), 40, 24),
            (333, 1, 4, (3, 4), 520, 264), (100, 1, 2, (16, 32), 72, 40), (2100, 2, 2, (7, 10), 200, 264),
            (25000, 1, 2, (1, 3), 72, 520), (1000, 1, 1, (1, 1), 264, 520), (17, 1, 1, (64, 64), 32, 8)]


@pytest.mark.parametrize("orders", ORDERS, ids="-".join)
@pytest.mark.parametrize("swiglu", [False, True], ids=["plain", "swiglu"])
@pytest.mark.parametrize("dtype", TYPES, ids=tid)
def test_product_orders(dtype, swiglu, orders):
    for T, grid in ((6, (4, 5)), (120, (1, 3))):
        _check_product(_case(T, 2, 2, grid, 72, 104, dtype, swiglu, orders))


@pytest.mark.parametrize("swiglu", [False, True], ids=["plain", "swiglu"])
@pytest.mark.parametrize("dtype", TYPES, ids=tid)
@pytest.mark.parametrize("shape", PRODUCTS, ids=lambda s: "x".join(map(str, s[:3])) + f"-{s[4]}-{s[5]}")
def test_product_sizes(shape, dtype, swiglu):
    _check_product(_case(*shape, dtype, swiglu))


@pytest.mark.parametrize("orders", ORDERS, ids="-".join)
@pytest.mark.parametrize("dtype", TYPES, ids=tid)
def test_product_gradient_orders(dtype, orders):
    for T, grid in ((6, (4, 5)), (120, (1, 3))):
        _check_product_back(_case(T, 2, 2, grid, 72, 104, dtype, False, orders))


# tiles of the weight gradients of every side, and their sums in parts
@pytest.mark.parametrize("dtype", TYPES, ids=tid)
@pytest.mark.parametrize("shape", PRODUCTS + [(700, 1, 1, (10, 20), 264, 264), (700, 1, 1, (5, 8), 264, 200),
                                              (6001, 1, 1, (1, 1), 72, 72), (3000, 1, 2, (1, 2), 136, 72)],
                         ids=lambda s: "x".join(map(str, s[:3])) + f"-{s[4]}-{s[5]}")
def test_product_gradient_sizes(shape, dtype):
    _check_product_back(_case(*shape, dtype))


# sizes at which the products take tiles of each side
@pytest.mark.parametrize("swiglu", [False, True], ids=["plain", "swiglu"])
@pytest.mark.parametrize("shape", [(9000, 1, 1, (2, 4), 264, 776), (4000, 1, 1, (4, 4), 264, 1032),
                                   (4000, 1, 1, (1, 1), 264, 1032), (4500, 1, 2, (4, 10), 264, 264)],
                         ids=lambda s: f"{s[0]}-{s[4]}-{s[5]}")
def test_product_tiles(shape, swiglu):
    for orders in (("token", "position"), ("task", "task")):
        _check_product(_case(*shape, BF16, swiglu, orders, seed=11))


@pytest.mark.parametrize("shape", [(9000, 1, 1, (2, 4), 776, 264), (4000, 1, 1, (4, 4), 1032, 264), (4000, 1, 1, (1, 1), 264, 264)],
                         ids=lambda s: f"{s[0]}-{s[4]}-{s[5]}")
def test_product_gradient_tiles(shape):
    for orders in (("position", "position"), ("task", "task")):
        _check_product_back(_case(*shape, BF16, False, orders, seed=12))


# dW's tiles of each side, its experts by rank over all XCDs, to and fro, or in order, whole and in parts
@pytest.mark.parametrize("orders", [("token", "position"), ("position", "task")], ids="-".join)
@pytest.mark.parametrize("shape", [(4000, 1, 1, (4, 10), 520, 520), (4000, 1, 1, (3, 5), 520, 776), (9000, 1, 1, (1, 1), 520, 776),
                                   (20000, 1, 1, (1, 3), 264, 520), (3000, 1, 1, (2, 4), 4104, 4104),
                                   (3000, 1, 1, (3, 8), 2056, 4104), (1500, 1, 2, (2, 13), 2056, 4104),
                                   (12000, 1, 1, (1, 1), 2056, 2056), (20000, 1, 1, (1, 2), 1288, 1544)],
                         ids=lambda s: f"{s[0]}-{s[3][0] * s[3][1]}-{s[4]}-{s[5]}")
def test_weight_gradient_tiles(shape, orders):
    _check_dw(_case(*shape, BF16, False, orders, seed=13, weights=False))


# tiles of 128 by rank, to and fro, in order and in parts, and long sums of few experts
@pytest.mark.parametrize("shape", [(1500, 1, 1, (3, 4), 520, 776), (9000, 1, 1, (4, 4), 1032, 520), (4000, 1, 1, (4, 5), 1032, 776),
                                   (30000, 1, 1, (1, 1), 520, 264), (65536, 1, 1, (2, 2), 1024, 1024)],
                         ids=lambda s: f"{s[0]}-{s[3][0] * s[3][1]}-{s[4]}-{s[5]}")
def test_weight_gradient_tiles_of_long_sums(shape):
    _check_dw(_case(*shape, BF16, False, ("token", "position"), seed=14, weights=False))


@pytest.mark.parametrize("dtype", TYPES, ids=tid)
@pytest.mark.parametrize("idx", ["first", "last", "one each", "empty between"])
def test_product_of_uneven_experts(idx, dtype):
    T, N = 300, 9
    ids = {"first": [0] * T, "last": [N - 1] * T, "one each": [i % N if i < N else 4 for i in range(T)],
           "empty between": [(i % 3) * 4 for i in range(T)]}[idx]
    for case_T in (T, 20):
        c = _case(case_T, 1, 1, (3, 3), 72, 136, dtype, idx=ids[:case_T])
        _check_product(c)
        _check_product_back(c)


@pytest.mark.parametrize("M", [20, 600])
@pytest.mark.parametrize("dtype", TYPES, ids=tid)
def test_positions_of_nobody(dtype, M):
    # positions behind the last expert's, and positions whose task does not exist, are not read and not written
    c = _case(M, 1, 1, (1, 4), 72, 40, dtype, orders=("task", "task"))
    full = _run(c, "omnimoe_grouped_product", c.x, c.w, shape=(M, c.n), orders=c.orders)
    o = c.offsets.clone()
    cut = M - M // 5
    o[o > cut] = cut
    lost = c.perm[cut:].clone()
    c.offsets = o
    c.x[lost.long()] = NAN
    c.dy[lost.long()] = NAN
    perm = c.perm.clone()
    c.perm[cut:] = 1 << 30
    gone = c.perm[3].clone()
    c.perm[3], c.x[gone.long()], c.dy[gone.long()] = -1, NAN, NAN
    got = _run(c, "omnimoe_grouped_product", c.x, c.w, shape=(M, c.n), orders=c.orders)
    kept = torch.ones(M, dtype=torch.bool, device="cuda")
    kept[lost.long()] = False
    kept[gone.long()] = False
    assert same_bits(got[kept], full[kept]) and bool(torch.isnan(got[~kept]).all())
    dx = _run(c, "omnimoe_grouped_product_dx", c.dy, c.w, shape=(M, c.k), orders=c.orders)
    assert bool(torch.isfinite(dx[kept]).all()) and bool(torch.isnan(dx[~kept]).all())
    dw = torch.empty_like(c.w)
    P.omnimoe_grouped_product_dw(c.D, c.q, c.x, c.dy, c.offsets, c.perm, dw)
    c.perm = perm
    x, dy = _by_position(c, c.x, "task"), _by_position(c, c.dy, "task")
    x[3], dy[3] = 0, 0
    x[cut:], dy[cut:] = 0, 0
    within(dw, *K.product_dw(x, dy, c.offsets, dtype), "dw")
    # rows by position on one side: its rows of lost tasks are not read either
    c = _case(M, 1, 1, (1, 4), 72, 40, dtype, orders=("position", "task"))
    gone = int(c.perm[3])
    c.perm[3], c.x[3], c.dy[gone] = M, NAN, NAN
    P.omnimoe_grouped_product_dw(c.D, c.q, c.x, c.dy, c.offsets, c.perm, dw)
    assert bool(torch.isfinite(dw).all())


GATES = [-400, -349, -200, -187, -180, -177, -150, -128, -110, -104, -100, -92, -89, -88.5, -88, -87, -80.5, -80, -79.5, -40,
         -1, 0, 1, 40, 88, 89, 100]


def _gated_case(shape, dtype, seed):
    """Rows of x that pick one value of every weight row, so that gate and up value are known exactly; gates from -400 to 100,
    up values from 2^-20 to 2^100."""
    c = _case(*shape, dtype, True, seed=seed)
    g = torch.Generator().manual_seed(seed)
    gate = torch.rand((c.N, c.n, c.k), generator=g) * 200 - 100
    gate.view(-1)[:27 * (gate.numel() // 27 // 3)].view(-1, 27)[:] = torch.tensor(GATES)
    up = torch.exp2(torch.randint(-20, 101, gate.shape, generator=g).float()) * (torch.rand(gate.shape, generator=g) + 0.5)
    c.w = torch.cat((gate, up), 1).to(dtype).cuda()
    c.x = torch.zeros((c.T, c.k), dtype=dtype, device="cuda")
    c.at = torch.arange(c.T, device="cuda") % c.k
    c.x[torch.arange(c.T, device="cuda"), c.at] = 1.0
    return c


def _check_gates(c, fn, weights, w):
    got = _run(c, fn, c.x, *weights, shape=(c.M, c.n), orders=c.orders)
    expert = torch.repeat_interleave(torch.arange(c.N, device="cuda"), (_ends(c)[1:] - _ends(c)[:-1]).long())
    rows = w[expert, :, c.at[c.perm.long() // c.hk]].to(F64)
    g, u = rows[:, :c.n], rows[:, c.n:]
    want = S.silu(g) * u
    # bf16's exponents: the constant's and the product's rounding are |g| 2^-24 each of the result; beside them one power (two
    # units of 2^-24; of the fourth root's four times) and up to five products, or a sum, a division and two products
    rel = ((2 * g.abs() if c.dtype is BF16 else 0) + 16) * S.U32
    r = S.unit(c.dtype)
    within(got, want, want.abs() * (rel * (1 + r) + r) + K.least(c.dtype), fn)


# few rows, and tiles of every side
@pytest.mark.parametrize("dtype", TYPES, ids=tid)
@pytest.mark.parametrize("shape", [(5, 1, 1, (1, 1), 72, 104), (200, 1, 1, (2, 3), 72, 104), (9000, 1, 1, (2, 4), 264, 776),
                                   (4000, 1, 1, (4, 4), 264, 1032), (4000, 1, 1, (1, 1), 264, 1032)],
                         ids=lambda s: f"{s[0]}-{s[3][0] * s[3][1]}-{s[4]}-{s[5]}")
def test_product_gates_at_their_ends(shape, dtype):
    c = _gated_case(shape, dtype, 91)
    _check_gates(c, "omnimoe_grouped_product", (c.w,), c.w)


@pytest.mark.parametrize("dtype", TYPES, ids=tid)
@pytest.mark.parametrize("shape", [(5, 1, 1, (1, 1), 96, 104), (70, 1, 2, (2, 3), 96, 104)], ids=["one", "six"])
def test_product4_gates_at_their_ends(shape, dtype):
    c = _gated_case(shape, dtype, 92)
    codes, scales, back = _store(c.D, c.q, c.w)
    _check_gates(c, "omnimoe_grouped_product4", (codes, scales), back)


@pytest.mark.parametrize("T", [24, 900])
@pytest.mark.parametrize("bad", [INF, NAN])
def test_product_keeps_what_is_not_finite_in_its_row(T, bad):
    c = _case(T, 1, 1, (1, 3), 136, 72, BF16, swiglu=True)
    clean = _check_product(c)
    p = 7
    c.x[int(c.perm[p]), 135] = bad
    got = _run(c, "omnimoe_grouped_product", c.x, c.w, shape=(c.M, c.n), orders=c.orders)
    others = torch.arange(c.M, device="cuda") != p
    assert same_bits(got[others], clean[others]) and not bool(torch.isfinite(got[p]).all())


def test_product_of_no_tokens():
    c = _case(0, 1, 1, (2, 2), 64, 64, BF16)
    P.omnimoe_grouped_product(c.D, c.q, None, c.w, None, None, None)
    dw = torch.full_like(c.w, 3.0)
    P.omnimoe_grouped_product_dw(c.D, c.q, None, None, None, None, dw)
    assert int(dw.count_nonzero()) == 0
    # no tokens: nothing is divided by H K, which has no 32-bit value here
    D = S.desc(0, 64, BF16, n_rows=64, n_cols=64, K=4096, H=1 << 20)
    dw = torch.full((4096, 8, 8), 3.0, dtype=BF16, device="cuda")
    P.omnimoe_grouped_product_dw(D, P.make_product(8, 8, False, "token", "task"), None, None, None, None, dw)
    assert int(dw.count_nonzero()) == 0


def test_product_rows_past_4_gib():
    # x by token past 2^32 bytes; the rows far behind are told apart
    T, k = 300000, 8192
    D = S.desc(T, 64, BF16, n_rows=1, n_cols=2, query_mode="shared")
    x = torch.zeros((T, k), dtype=BF16, device="cuda")
    x[-1, -1], x[T // 2, 3] = 2.0, 3.0
    w = torch.zeros((2, 8, k), dtype=BF16, device="cuda")
    w[0, 5, 3], w[1, 6, -1] = 1.0, 1.0
    offsets = torch.tensor([0, T // 2 + 1, T], dtype=torch.int32, device="cuda")
    perm = torch.arange(T, dtype=torch.int32, device="cuda")
    q = P.make_product(k, 8, False, "token", "task")
    y = torch.empty((T, 8), dtype=BF16, device="cuda")
    P.omnimoe_grouped_product(D, q, x, w, offsets, perm, y)
    assert float(y[T // 2, 5]) == 3 and float(y[-1, 6]) == 2 and int(y.count_nonzero()) == 2
    dw = torch.empty_like(w)
    P.omnimoe_grouped_product_dw(D, q, x, torch.ones_like(y), offsets, perm, dw)
    assert bool((dw[0, :, 3] == 3).all()) and bool((dw[1, :, -1] == 2).all()) and int(dw.count_nonzero()) == 16


def _check_rows(x, w, experts, y, at, swiglu=False):
    """Positions `at` of y, whose rows of x lie there too, by themselves."""
    one = torch.tensor([0, 1], device="cuda")
    for p, e in zip(at, experts):
        want, bound = K.product(x[p:p + 1].to(F64), w[e:e + 1], one, swiglu, BF16)
        within(y[p:p + 1], want, bound, f"position {p}")


def _no_nan(y, rows):
    assert not any(bool(torch.isnan(y[i:i + rows]).any()) for i in range(0, len(y), rows))


def test_few_rows_past_2_32_threads():
    T, N, n = 4096, 4096, 65536
    D = S.desc(T, 64, BF16, n_rows=64, n_cols=64, K=2, query_mode="shared")
    x, w = S.randn(1, 2 * T, 8, dtype=BF16), torch.randn((N, 2 * n, 8), dtype=BF16, device="cuda")
    offsets = torch.arange(0, 2 * N + 1, 2, dtype=torch.int32, device="cuda")
    y = torch.full((2 * T, n), NAN, dtype=BF16, device="cuda")
    P.omnimoe_grouped_product(D, P.make_product(8, n, True, "position", "position"), x, w, offsets, None, y)
    at = [0, 1, 2, 4095, 6000, 7279, 7280, 7281, 7282, 8000, 8190, 8191]
    _check_rows(x, w, [p // 2 for p in at], y, at, True)
    _no_nan(y, 2048)


def test_tiles_past_2_32_threads():
    T, H = 4194307, 128
    M = T * H * 2
    D = S.desc(T, 64, BF16, n_rows=1, n_cols=2, H=H, K=2, query_mode="shared")
    x = torch.ones((M, 8), dtype=BF16, device="cuda")
    x[M - 1], x[M // 2], x[0] = 3.0, 5.0, 7.0
    w = S.randn(3, 2, 8, 8, dtype=BF16)
    offsets = torch.tensor([0, M // 2 + 100, M], dtype=torch.int32, device="cuda")
    y = torch.full((M, 8), NAN, dtype=BF16, device="cuda")
    P.omnimoe_grouped_product(D, P.make_product(8, 8, False, "position", "position"), x, w, offsets, None, y)
    at = [0, 1, M // 2, M // 2 + 99, M // 2 + 100, M - 129, M - 2, M - 1]
    _check_rows(x, w, [int(p >= M // 2 + 100) for p in at], y, at)
    assert bool((y[1:M // 2] == y[1]).all()) and bool((y[M // 2 + 100:M - 1] == y[M - 2]).all())


# ------------------------------------------------------------------ 4-bit weights

def _store(D, q, w):
    codes = Guarded((*w.shape[:2], w.shape[2] // 2), torch.uint8)
    scales = Guarded((*w.shape[:2], w.shape[2] // 32), torch.uint8)
    back = Guarded(tuple(w.shape), w.dtype)
    P.omnimoe_weights4_store(D, q, w, codes.t, scales.t)
    P.omnimoe_weights4_load(D, q, codes.t, scales.t, back.t)
    torch.cuda.synchronize()
    for b in (codes, scales, back):
        b.check()
    return codes.t, scales.t, back.t


@pytest.mark.parametrize("swiglu", [False, True], ids=["plain", "swiglu"])
@pytest.mark.parametrize("dtype", TYPES, ids=tid)
def test_weights4_are_exact(dtype, swiglu):
    N, n, k = 3, 40, 352
    w = S.randn(1, N, n * (1 + swiglu), k, dtype=dtype) * torch.exp2(S.randn(2, N, n * (1 + swiglu), 1, scale=4.0)).to(dtype)
    edge = torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -5.0, 0.2500001, 4.9999, 0.0, -0.0, 6.0])
    w[0, 0, :16] = edge.to(dtype)
    w[0, 1, :32] = 0
    w[0, 2, :32] = torch.finfo(dtype).max
    w[0, 3, :32] = 2.0 ** -126
    w[0, 4, 5], w[0, 5, 40], w[0, 6, 64] = INF, NAN, -INF
    D = S.desc(1, 64, dtype, n_rows=1, n_cols=N)
    codes, scales, back = _store(D, P.make_product(k, n, swiglu), w)
    want, s = K.quantise4(w)
    assert torch.equal(scales, s)
    fill = lambda t: torch.nan_to_num(t.to(F64), nan=1234.5)  # noqa: E731
    assert torch.equal(fill(back), fill(want)) and torch.equal(fill(K.dequantise4(codes, scales)), fill(want))


def _case4(*a, **kw):
    c = _case(*a, **kw)
    codes, scales, back = _store(c.D, c.q, c.w)
    assert torch.equal(back.to(F64), K.dequantise4(codes, scales))
    c.weights, c.back = (codes, scales), back
    return c


PRODUCTS4 = [(1, 1, 1, (1, 1), 32, 8), (1, 1, 8, (8, 8), 2048, 72), (16, 1, 8, (8, 8), 160, 264), (5, 2, 3, (2, 3), 96, 24),
             (333, 1, 4, (3, 4), 544, 264), (7, 1, 1, (1, 1), 2080, 2056), (40, 1, 1, (1, 1), 640, 40),
             (17, 1, 1, (64, 64), 32, 8)]


@pytest.mark.parametrize("swiglu", [False, True], ids=["plain", "swiglu"])
@pytest.mark.parametrize("dtype", TYPES, ids=tid)
@pytest.mark.parametrize("shape", PRODUCTS4, ids=lambda s: "x".join(map(str, s[:3])) + f"-{s[4]}-{s[5]}")
def test_product4_sizes(shape, dtype, swiglu):
    c = _case4(*shape, dtype, swiglu)
    _check_product(c, "omnimoe_grouped_product4", c.weights, c.back)


@pytest.mark.parametrize("orders", ORDERS, ids="-".join)
@pytest.mark.parametrize("dtype", TYPES, ids=tid)
def test_product4_orders(dtype, orders):
    c = _case4(11, 2, 2, (4, 5), 96, 104, dtype, True, orders)
    _check_product(c, "omnimoe_grouped_product4", c.weights, c.back)


@pytest.mark.parametrize("dtype", TYPES, ids=tid)
def test_product4_with_every_code_and_scale(dtype):
    # rows of x that pick one value of every weight row: each code at each scale that store writes, and the byte of NaN
    n, k = 256, 32
    codes = torch.randint(0, 256, (1, n, k // 2), generator=torch.Generator().manual_seed(5), dtype=torch.uint8).cuda()
    scales = torch.arange(n, dtype=torch.uint8).view(1, n, 1).cuda()
    scales[0, :2], scales[0, 253:255] = 2, 252
    D, q = S.desc(k, 64, dtype, n_rows=1, n_cols=1), P.make_product(k, n)
    x = torch.eye(k, dtype=dtype, device="cuda")
    y = torch.empty((k, n), dtype=dtype, device="cuda")
    P.omnimoe_grouped_product4(D, q, x, codes, scales, None, None, y)
    want = K.dequantise4(codes, scales)[0].t()
    assert torch.equal(torch.nan_to_num(y.to(F64), nan=1234.5), torch.nan_to_num(want, nan=1234.5))
    assert bool(torch.isnan(y[:, 255]).all()) and bool(torch.isfinite(y[:, :255]).all())


def test_product4_past_2_32_threads():
    M, n = 131088, 65536
    D, q = S.desc(M, 64, BF16, n_rows=1, n_cols=1, K=1, query_mode="shared"), P.make_product(32, n, True, "position", "position")
    codes, scales, w = _store(D, q, S.randn(5, 1, 2 * n, 32, dtype=BF16))
    x, y = S.randn(6, M, 32, dtype=BF16), torch.full((M, n), NAN, dtype=BF16, device="cuda")
    P.omnimoe_grouped_product4(D, q, x, codes, scales, None, None, y)
    at = [0, 17, 65535, 131055, 131056, 131071, 131072, 131087]
    _check_rows(x, w, [0] * len(at), y, at, True)
    _no_nan(y, 8192)


def test_product4_positions_of_nobody():
    c = _case4(20, 1, 1, (1, 4), 96, 40, BF16, orders=("task", "task"))
    full = _run(c, "omnimoe_grouped_product4", c.x, *c.weights, shape=(c.M, c.n), orders=c.orders)
    cut = c.M - 4
    c.offsets = c.offsets.clamp(max=cut)
    lost = c.perm[cut:].long()
    gone = int(c.perm[2])
    c.perm[2] = c.M
    got = _run(c, "omnimoe_grouped_product4", c.x, *c.weights, shape=(c.M, c.n), orders=c.orders)
    kept = torch.ones(c.M, dtype=torch.bool, device="cuda")
    kept[lost], kept[gone] = False, False
    assert same_bits(got[kept], full[kept]) and bool(torch.isnan(got[~kept]).all())


# ------------------------------------------------------------------ streams, graphs, side by side

def _all_calls():
    """Every entry point once, with its inputs, as (launch(stream), outputs)."""
    calls = []
    for T, d, dtype in ((70, 520, BF16), (5, 2048, F32)):
        i = _join_inputs(T, d, dtype, "channel")
        x_out, n = torch.empty_like(i.x), torch.empty_like(i.x)
        calls.append((lambda st, i=i, x_out=x_out, n=n: P.omnimoe_block_join(
            i.D, i.eps, i.x, i.y, i.gate, i.w_out, i.scale, i.w_in, x_out, n, stream=st), [x_out, n]))
        o = [torch.empty_like(t) for t in (i.x, i.y, i.gate, i.w_out, i.scale, i.w_in)]
        ws = torch.empty(P.omnimoe_block_join_backward_workspace_size(i.D), dtype=torch.uint8, device="cuda")
        kept = _join(i)[0]
        calls.append((lambda st, i=i, o=o, ws=ws, kept=kept: P.omnimoe_block_join_backward(
            i.D, i.eps, kept, i.y, i.gate, i.w_out, i.scale, i.w_in, i.dx_out, i.dn, *o, ws=ws, stream=st), o))
    for c in (_case(9, 1, 4, (4, 4), 264, 136, BF16, True), _case(700, 1, 2, (2, 3), 264, 136, BF16, True),
              _case(50, 1, 2, (2, 3), 72, 40, F32, False, ("task", "task"))):
        y = torch.zeros((c.M, c.n), dtype=c.dtype, device="cuda")
        calls.append((lambda st, c=c, y=y: P.omnimoe_grouped_product(c.D, c.q, c.x, c.w, c.offsets, c.perm, y, stream=st), [y]))
    c = _case(3000, 1, 1, (1, 2), 72, 136, BF16, False, ("task", "task"))
    dx, dw = torch.zeros((c.M, c.k), dtype=BF16, device="cuda"), torch.zeros_like(c.w)
    ws = torch.empty(max(256, P.omnimoe_grouped_product_dw_workspace_size(c.D, c.q)), dtype=torch.uint8, device="cuda")
    calls.append((lambda st: P.omnimoe_grouped_product_dx(c.D, c.q, c.dy, c.w, c.offsets, c.perm, dx, stream=st), [dx]))
    calls.append((lambda st: P.omnimoe_grouped_product_dw(c.D, c.q, c.x, c.dy, c.offsets, c.perm, dw, ws=ws, stream=st), [dw]))
    f = _case4(9, 1, 4, (4, 4), 352, 136, BF16, True)
    y4 = torch.zeros((f.M, f.n), dtype=BF16, device="cuda")
    calls.append((lambda st: P.omnimoe_grouped_product4(f.D, f.q, f.x, *f.weights, f.offsets, f.perm, y4, stream=st), [y4]))
    codes, scales, back = torch.zeros_like(f.weights[0]), torch.zeros_like(f.weights[1]), torch.zeros_like(f.w)
    calls.append((lambda st: P.omnimoe_weights4_store(f.D, f.q, f.w, codes, scales, stream=st), [codes, scales]))
    calls.append((lambda st: P.omnimoe_weights4_load(f.D, f.q, *f.weights, back, stream=st), [back]))
    return calls


def _bytes(outs):
    return [t.contiguous().view(torch.uint8).clone() for t in outs]


def test_calls_on_other_streams_and_side_by_side():
    calls = _all_calls()
    first = []
    for launch, outs in calls:
        launch(None)
        torch.cuda.synchronize()
        first.append(_bytes(outs))
        for t in outs:
            t.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for n, (launch, _) in enumerate(calls):  # each call on a stream of its own, all in flight
        launch(streams[n % 3])
    torch.cuda.synchronize()
    for (_, outs), want in zip(calls, first):
        assert all(torch.equal(a, b) for a, b in zip(_bytes(outs), want))
    with torch.cuda.stream(streams[0]):  # the current stream
        for launch, _ in calls:
            launch(None)
    torch.cuda.synchronize()
    for (_, outs), want in zip(calls, first):
        assert all(torch.equal(a, b) for a, b in zip(_bytes(outs), want))


def test_calls_in_a_graph():
    calls = _all_calls()
    first = []
    for launch, outs in calls:
        launch(None)
        torch.cuda.synchronize()
        first.append(_bytes(outs))
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        for launch, _ in calls:
            launch(None)
    for replay in range(4):
        for _, outs in calls:
            for t in outs:
                t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for n, ((launch, outs), want) in enumerate(zip(calls, first)):
            assert all(torch.equal(a, b) for a, b in zip(_bytes(outs), want)), (replay, n)
        calls[replay][0](None)  # the program's own eager work between the replays


# ------------------------------------------------------------------ as they are used

def _experts_step(T, d, f, Kk, grid, dtype, seed=0):
    """A block of a model: the joint's norm, the router and its schedule, experts with matrices of their own."""
    N, M = grid[0] * grid[1], T * Kk
    s = SimpleNamespace(T=T, d=d, f=f, Kk=Kk, N=N, M=M, dtype=dtype,
                        D=S.desc(T, d, dtype, n_rows=grid[0], n_cols=grid[1], d_key=d // 2, K=Kk),
                        x=S.randn(seed, T, d, dtype=dtype), w_norm=S.randn(seed + 1, d) * 0.1 + 1,
                        keys_row=S.randn(seed + 2, 1, grid[0], d // 2, scale=d ** -0.5, dtype=dtype),
                        keys_col=S.randn(seed + 3, 1, grid[1], d // 2, scale=d ** -0.5, dtype=dtype),
                        w_gu=S.randn(seed + 4, N, 2 * f, d, scale=d ** -0.5, dtype=dtype),
                        w_down=S.randn(seed + 5, N, d, f, scale=f ** -0.5, dtype=dtype),
                        scale=S.randn(seed + 6, d) * 0.1 + 0.5, gate=S.randn(seed + 7, T, dtype=dtype))
    new = lambda shape, dt: torch.empty(shape, dtype=dt, device="cuda")  # noqa: E731
    s.n, s.x_out, s.n_next = (new((T, d), dtype) for _ in range(3))
    s.idx, s.gates = new((T, 1, Kk), torch.int32), new((T, 1, Kk), F32)
    s.perm, s.offsets = new((M,), torch.int32), new((N + 1,), torch.int32)
    s.active, s.ends, s.count = new((min(M, N),), torch.int32), new((min(M, N) + 1,), torch.int32), new((1,), torch.int32)
    P.omnimoe_block_join(s.D, 1e-6, s.x, None, None, None, None, s.w_norm, None, s.n)
    P.omnimoe_route(s.D, s.n, s.keys_row, s.keys_col, s.idx, s.gates)
    P.omnimoe_schedule(s.D, s.idx, s.perm, s.active, s.ends, s.count, s.offsets)
    return s


def _experts_plain(n, gates, s, w_gu, w_down):
    """sum over a token's experts of gate W_down (silu(G n) (U n)), differentiable, in 64 bits."""
    y = torch.zeros((s.T, s.d), dtype=F64, device="cuda")
    idx = s.idx.view(s.T, s.Kk)
    for e in range(s.N):
        t, k = (idx == e).nonzero(as_tuple=True)
        if t.numel():
            h = n[t] @ w_gu[e].t()
            a = torch.nn.functional.silu(h[:, :s.f]) * h[:, s.f:]
            y = y.index_add(0, t, gates[t, k, None] * (a @ w_down[e].t()))
    return y


def _rel(got, want):
    return float((got.to(F64) - want).norm() / want.norm())


@pytest.mark.parametrize("dtype", TYPES, ids=tid)
def test_training_step_of_a_block(dtype):
    s = _experts_step(200, 128, 96, 2, (3, 4), dtype)
    T, d, f, Kk, M = s.T, s.d, s.f, s.Kk, s.M
    new = lambda shape, dt=dtype: torch.empty(shape, dtype=dt, device="cuda")  # noqa: E731
    gu = P.make_product(d, 2 * f, False, "token", "position")
    down = P.make_product(f, d, False, "position", "task")
    h, z = new((M, 2 * f)), new((M, d))
    P.omnimoe_grouped_product(s.D, gu, s.n, s.w_gu, s.offsets, s.perm, h)
    a = (torch.nn.functional.silu(h[:, :f].float()) * h[:, f:].float()).to(dtype)
    fused = new((M, f))
    P.omnimoe_grouped_product(s.D, P.make_product(d, f, True, "token", "position"), s.n, s.w_gu, s.offsets, s.perm, fused)
    P.omnimoe_grouped_product(s.D, down, a, s.w_down, s.offsets, s.perm, z)
    gates = s.gates.view(T, Kk)
    y = (z.view(T, Kk, d).float() * gates[:, :, None]).sum(1)
    P.omnimoe_block_join(s.D, 1e-6, s.x, y, s.gate, s.w_norm, s.scale, s.w_norm, s.x_out, s.n_next)
    # the way back
    dx_out, dn = S.randn(90, T, d, dtype=dtype), S.randn(91, T, d, dtype=dtype)
    dx, dy, dgate = new((T, d)), new((T, d), F32), torch.empty_like(s.gate)
    dw_out, dscale, dw_in = (new((d,), F32) for _ in range(3))
    P.omnimoe_block_join_backward(s.D, 1e-6, s.x_out, y, s.gate, s.w_norm, s.scale, s.w_norm, dx_out, dn, dx, dy, dgate,
                                  dw_out, dscale, dw_in)
    dz = (dy[:, None] * gates[:, :, None]).to(dtype).view(M, d)
    dgates = (z.view(T, Kk, d).float() * dy[:, None]).sum(2)
    da, dw_down = new((M, f)), torch.empty_like(s.w_down)
    P.omnimoe_grouped_product_dx(s.D, down, dz, s.w_down, s.offsets, s.perm, da)
    P.omnimoe_grouped_product_dw(s.D, down, a, dz, s.offsets, s.perm, dw_down)
    g, u = h[:, :f].float(), h[:, f:].float()
    dh = torch.cat((da.float() * u * S.dsilu(g), da.float() * S.silu(g)), 1).to(dtype)
    back, dw_gu = P.make_product(d, 2 * f, False, "task", "position"), torch.empty_like(s.w_gu)
    rows = new((M, d))
    P.omnimoe_grouped_product_dx(s.D, back, dh, s.w_gu, s.offsets, s.perm, rows)
    P.omnimoe_grouped_product_dw(s.D, gu, s.n, dh, s.offsets, s.perm, dw_gu)
    dn1 = rows.view(T, Kk, d).float().sum(1).to(dtype)
    first, dw_first = new((T, d)), new((d,), F32)
    P.omnimoe_block_join_backward(s.D, 1e-6, s.x, None, None, None, None, s.w_norm, dx, dn1, first, None, None, None, None,
                                  dw_first)
    # the same in 64 bits, gates of the GPU's routing
    v = {k: getattr(s, k).to(F64).requires_grad_() for k in ("x", "w_gu", "w_down", "scale", "gate")}
    G = gates.to(F64).requires_grad_()
    w1, w2, w3 = (s.w_norm.to(F64).requires_grad_() for _ in range(3))
    _, n = K.join(v["x"], None, None, None, None, w1, 1e-6)
    yy = _experts_plain(n, G, s, v["w_gu"], v["w_down"])
    xo, nn = K.join(v["x"], yy, v["gate"][:, None], w2, v["scale"], w3, 1e-6)
    ((xo * dx_out.to(F64)).sum() + (nn * dn.to(F64)).sum()).backward()
    # At most eight values in a row are rounded to the layer's type between an input and a result (n, h, a, z or dx, dz, da,
    # dh, the result), each by half a step of itself; fp32 layers: sums of up to 400 products, 2 * 400 * 2^-24 each.
    most = 8 * S.unit(dtype) if dtype is BF16 else 8 * S.gamma(400)
    pairs = dict(fused=(fused, a.to(F64)), x_out=(s.x_out, xo), n=(s.n_next, nn), dx=(first, v["x"].grad),
                 dw_gu=(dw_gu, v["w_gu"].grad), dw_down=(dw_down, v["w_down"].grad), dscale=(dscale, v["scale"].grad),
                 dgate=(dgate, v["gate"].grad), dgates=(dgates, G.grad), dw_first=(dw_first, w1.grad), dw_out=(dw_out, w2.grad),
                 dw_in=(dw_in, w3.grad))
    for k, (got, want) in pairs.items():
        assert _rel(got, want.detach()) <= most, (k, _rel(got, want.detach()), most)


@pytest.mark.parametrize("T", [1, 13])
def test_decode_step_with_4_bit_experts(T):
    dtype = BF16
    s = _experts_step(T, 256, 160, 4, (4, 4), dtype, seed=5)
    d, f, M = s.d, s.f, s.M
    up, down = P.make_product(d, f, True, "token", "position"), P.make_product(f, d, False, "position", "task")
    c_gu, s_gu, w_gu = _store(s.D, up, s.w_gu)
    c_dn, s_dn, w_dn = _store(s.D, down, s.w_down)
    a, z = torch.empty((M, f), dtype=dtype, device="cuda"), torch.empty((M, d), dtype=dtype, device="cuda")
    P.omnimoe_grouped_product4(s.D, up, s.n, c_gu, s_gu, s.offsets, s.perm, a)
    P.omnimoe_grouped_product4(s.D, down, a, c_dn, s_dn, s.offsets, s.perm, z)
    y = (z.view(T, s.Kk, d).float() * s.gates.view(T, s.Kk, 1)).sum(1)
    P.omnimoe_block_join(s.D, 1e-6, s.x, y, s.gate, s.w_norm, s.scale, s.w_norm, s.x_out, s.n_next)
    yy = _experts_plain(s.n.to(F64), s.gates.view(T, s.Kk).to(F64), s, w_gu.to(F64), w_dn.to(F64))
    xo, nn = K.join(s.x.to(F64), yy, s.gate.to(F64)[:, None], s.w_norm.to(F64), s.scale.to(F64), s.w_norm.to(F64), 1e-6)
    # a, z and the result are rounded to bf16 in a row
    assert _rel(s.x_out, xo) <= 3 * S.unit(dtype) and _rel(s.n_next, nn) <= 3 * S.unit(dtype)
