"""The operators of include/omnimoe_ffn.h on the GPU against plain 64-bit forms, within bounds derived from their
roundings (ffn_support), at the sizes, values and orders where they could go wrong; their use under graph capture, on
other streams and side by side; and a training and a decode step in which they run with the routed layer's."""
import sys
from types import SimpleNamespace

import pytest

import synth  # noqa: F401  (the package's root on the path)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
import ffn_support as S  # noqa: E402
import paper_2602_05711_amd as P  # noqa: E402
from paper_2602_05711_amd import binding as B  # noqa: E402

BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
TYPES = [BF16, F32]
tid = {BF16: "bf16", F32: "f32"}.get


def within(got, want, bound, what):
    got = got.to(F64)
    assert torch.isfinite(got).all(), what
    over = (got - want).abs() - bound
    worst = float(over.max()) if over.numel() else 0.0
    assert worst <= 0, f"{what}: {worst:.3e} over its bound {float(bound.reshape(-1)[over.argmax()]):.3e}"


class Guarded:
    """A tensor of `shape` with sentinel bytes after it, which no call may change."""

    def __init__(self, shape, dtype):
        n = 1
        for s in shape:
            n *= s
        size = torch.empty((), dtype=dtype).element_size()
        self.raw = torch.full((n * size + 512,), 0xA5, dtype=torch.uint8, device="cuda")
        self.n = n * size
        self.t = self.raw[:self.n].view(dtype).view(shape)

    def check(self):
        assert bool((self.raw[self.n:] == 0xA5).all()), "written past the end"


# ------------------------------------------------------------------ checkpoint

def _store(x):
    T, d = x.shape
    D = S.desc(T, d, x.dtype)
    codes, scales = Guarded((T, d), torch.uint8), Guarded((T, -(-d // 32)), torch.uint8)
    back = Guarded((T, d), x.dtype)
    P.omnimoe_checkpoint_store(D, x, codes.t, scales.t)
    P.omnimoe_checkpoint_load(D, codes.t, scales.t, back.t)
    torch.cuda.synchronize()
    for b in (codes, scales, back):
        b.check()
    return codes.t, scales.t, back.t


def _same(a, b):
    return torch.equal(torch.nan_to_num(a, nan=12345.0), torch.nan_to_num(b, nan=12345.0))


@pytest.mark.parametrize("dtype", TYPES, ids=tid)
@pytest.mark.parametrize("T,d", [(1, 8), (1, 2048), (3, 40), (7, 32), (65, 520), (333, 1000), (2, 4096), (4097, 64)])
def test_checkpoint_is_exact(T, d, dtype):
    x = S.randn(T + d, T, d, dtype=dtype) * torch.exp2(S.randn(1, 1, d, scale=3.0)).to(dtype)
    codes, scales, back = _store(x)
    want, s = S.quantise(x)
    assert torch.equal(scales, s) and torch.equal(back.to(F64), want)
    assert _same(S.dequantise(codes, scales), want)


def test_checkpoint_of_every_bf16_value():
    # all 2^16 patterns, in blocks of neighbours (one binade each), and in blocks that hold 1, so that the small ones sink
    bits = torch.arange(65536, dtype=torch.int32, device="cuda").to(torch.int16)
    x = bits.view(BF16).view(-1, 256)
    for v in (x, torch.cat((x.reshape(-1)[:2114 * 31].view(-1, 31), torch.ones(2114, 1, dtype=BF16, device="cuda")), 1).view(1057, 64)):
        v = v.contiguous()
        codes, scales, back = _store(v)
        want, s = S.quantise(v)
        assert torch.equal(scales, s)
        assert _same(S.dequantise(codes, scales), want)
        # what comes back in bf16 is the value itself (bf16 has every e4m3 value times 2^s but the tiniest
        # and past its largest)
        most = torch.finfo(BF16).max
        assert _same(back.to(F64), want.clamp(-most, most).to(F32).to(BF16).to(F64))


def test_checkpoint_ties_zeros_and_extremes():
    eps = 2.0 ** -20
    row = [448.0, 1.0625, 1.1875, 1.0625 + eps, 1.0625 - eps, 2.0 ** -7 * 1.5, 2.0 ** -9, 2.0 ** -10, 2.0 ** -10 + 2.0 ** -30,
           3 * 2.0 ** -10, -0.0, 0.0, 447.9, 432.0, 416.0, 17.0]
    x = torch.zeros(6, 64, dtype=F32)
    x[0, :16] = torch.tensor(row)
    x[1, :16] = torch.tensor(row) * 2.0 ** -100
    x[2, 0], x[2, 33] = 3.4e38, 1e-45            # the largest exponent, a subnormal alone in its block
    x[3, 5], x[3, 40], x[3, 41] = float("inf"), float("nan"), 3.0
    x[4, :32] = 448.0 * 1.0000001               # just over a power's reach
    x[5, 31] = 2.0 ** -126
    x = x.cuda()
    codes, scales, back = _store(x)
    want, s = S.quantise(x)
    most = torch.finfo(F32).max
    assert torch.equal(scales, s) and _same(back.to(F64), want.clamp(-most, most).to(F32).to(F64))
    assert float(back[2, 0]) == most
    assert scales[2].tolist() == [247, 0] and codes[3, 5].item() & 127 == 127


def test_checkpoint_of_a_long_batch():
    # rows past 2^31 bytes: one block is told apart far behind
    T, d = 300000, 8192
    x = torch.zeros((T, d), dtype=BF16, device="cuda")
    x[-1, -32:] = torch.arange(32, device="cuda").to(BF16)
    x[T // 2, 17] = 5.0
    codes, scales, back = _store(x)
    assert torch.equal(back[-1], S.quantise(x[-1:])[0][0].to(BF16)) and back[T // 2, 17] == 5.0
    assert int(codes[:T // 2].count_nonzero()) == 0 and scales[-1, -1] != 0


# ------------------------------------------------------------------ the shared branch's way back

def _backward_inputs(T, d, f, dtype, seed=0):
    x = S.randn(seed, max(T, 1), d)[:T]
    D = S.desc(T, d, dtype)
    codes, scales = torch.zeros((T, d), dtype=torch.uint8, device="cuda"), torch.zeros((T, -(-d // 32)), dtype=torch.uint8, device="cuda")
    P.omnimoe_checkpoint_store(D, x.to(dtype).contiguous(), codes, scales)
    return SimpleNamespace(D=D, codes=codes, scales=scales, w_gu=S.randn(seed + 1, 2 * f, d, scale=d ** -0.5, dtype=dtype),
                           w_down=S.randn(seed + 2, d, f, scale=f ** -0.5, dtype=dtype),
                           dy=S.randn(seed + 3, max(T, 1), d)[:T], dx_in=S.randn(seed + 4, max(T, 1), d)[:T], T=T, d=d, f=f,
                           dtype=dtype)


def _backward(i, dx_in=True, stream=None, guarded=False):
    dx, dwg, dwd = Guarded((i.T, i.d), i.dtype), Guarded((2 * i.f, i.d), i.dtype), Guarded((i.d, i.f), i.dtype)
    ws = Guarded((P.omnimoe_shared_mlp_backward_workspace_size(i.D, i.f),), torch.uint8)
    ws.t.fill_(0xFF)  # NaN in every type: nothing may be read before it is written
    P.omnimoe_shared_mlp_backward(i.D, i.f, i.codes, i.scales, i.w_gu, i.w_down, i.dy, i.dx_in if dx_in else None, dx.t,
                                  dwg.t, dwd.t, ws=ws.t, stream=stream)
    torch.cuda.synchronize()
    for b in (dx, dwg, dwd, ws):
        b.check()
    return dx.t, dwg.t, dwd.t


SHAPES = [(1, 8, 8), (1, 64, 64), (2, 72, 40), (63, 64, 128), (64, 128, 64), (65, 520, 24), (100, 40, 520), (129, 2048, 8),
          (257, 256, 264), (1000, 520, 520), (4093, 136, 72),
          (1, 40, 2056), (33, 72, 4104), (140, 520, 1400)]  # dx in parts
# bf16 only: tiles of 256 (hidden values, dx and weight gradients), whole and ragged, their rows and columns past the end
LARGE = [(6144, 64, 1024), (6100, 72, 1032), (12288, 1024, 1024), (12200, 1000, 1032)]
# and tiles of 128: of dx and the weight gradients, of the hidden values, of both; dx's of 256 beside the others
MIDDLE = [(2048, 1024, 128), (2000, 1032, 264), (4093, 72, 1000), (4096, 1024, 1024), (4090, 1000, 1016), (6100, 2040, 264)]


@pytest.mark.parametrize("T,d,f,dtype", [s + (t,) for s in SHAPES for t in TYPES] + [s + (BF16,) for s in LARGE + MIDDLE],
                         ids=lambda v: tid(v) if v in TYPES else str(v))
def test_backward(T, d, f, dtype):
    print(f"[backward] T={T} d={d} d_ff={f} {dtype}", file=sys.stderr, flush=True)
    i = _backward_inputs(T, d, f, dtype, seed=T + d + f)
    x = S.dequantise(i.codes, i.scales)
    args = (x, i.w_gu.to(F64), i.w_down.to(F64), i.dy.to(F64))
    want, bound = S.mlp_backward_bounds(*args, i.dx_in.to(F64), dtype)
    got = _backward(i)
    for g, w, b, name in zip(got, want, bound, ("dx", "dw_gu", "dw_down")):
        within(g, w, b, name)
    again = _backward(i)
    assert all(torch.equal(a, b) for a, b in zip(got, again)), "two runs differ"
    if T < 2000:
        want, bound = S.mlp_backward_bounds(*args, torch.zeros_like(x), dtype)
        within(_backward(i, dx_in=False)[0], want[0], bound[0], "dx without dx_in")


def test_backward_matches_differences():
    # the directional derivative of L = sum(dy MLP(x)) in 64 bits along random directions of the three inputs
    i = _backward_inputs(200, 96, 160, BF16, seed=5)
    x, wg, wd, dy = S.dequantise(i.codes, i.scales), i.w_gu.to(F64), i.w_down.to(F64), i.dy.to(F64)
    zero = torch.zeros_like(x)
    _, bound = S.mlp_backward_bounds(x, wg, wd, dy, zero, BF16)
    got = _backward(i, dx_in=False)

    def loss(a, b, c):
        h = a @ b.t()
        return float((dy * ((S.silu(h[:, :i.f]) * h[:, i.f:]) @ c.t())).sum())

    for k, v in enumerate((x, wg, wd)):
        to = S.randn(50 + k, *v.shape).to(F64)
        args = [x, wg, wd]
        h = 1e-5
        args[k] = v + h * to
        up = loss(*args)
        args[k] = v - h * to
        slope = (up - loss(*args)) / (2 * h)
        mine = float((got[k].to(F64) * to).sum())
        # the kernel's bound along the direction, and the difference's own error (2^-52 |loss| / h, h^2)
        assert abs(slope - mine) <= float((bound[k] * to.abs()).sum()) + 1e-6 * (1 + abs(slope) + abs(up))


@pytest.mark.parametrize("dtype", TYPES, ids=tid)
def test_backward_of_dy_past_the_largest_bf16(dtype):
    # fp32's largest value and one a little below it round to infinity in bf16; as two bf16 values they are kept to 2^-17
    i = _backward_inputs(3, 64, 72, dtype, seed=17)
    i.w_gu *= 2.0 ** -5
    i.w_down[5] *= 2.0 ** -20
    i.w_down[7] *= 2.0 ** -20
    i.dy[0, 5], i.dy[1, 7] = torch.finfo(F32).max, -(2.0 ** 128 - 2.0 ** 118)
    want, bound = S.mlp_backward_bounds(S.dequantise(i.codes, i.scales), i.w_gu.to(F64), i.w_down.to(F64), i.dy.to(F64),
                                        i.dx_in.to(F64), dtype)
    for g, w, b, name in zip(_backward(i), want, bound, ("dx", "dw_gu", "dw_down")):
        within(g, w, b, name)


def test_backward_of_no_tokens():
    for dtype in TYPES:
        i = _backward_inputs(0, 64, 40, dtype)
        dwg, dwd = torch.ones_like(i.w_gu), torch.ones_like(i.w_down)
        st = B.load_library().omnimoe_shared_mlp_backward(
            B.ctypes.byref(i.D), i.f, None, None, B._ptr(i.w_gu), B._ptr(i.w_down), None, None, None, B._ptr(dwg),
            B._ptr(dwd), None, 0, B._stream(None))
        torch.cuda.synchronize()
        assert st == 0 and not dwg.any() and not dwd.any()


def test_backward_in_place_fp32():
    i = _backward_inputs(77, 64, 72, F32)
    want = _backward(i)[0]
    dx, dwg, dwd = i.dx_in.clone(), torch.empty_like(i.w_gu), torch.empty_like(i.w_down)
    P.omnimoe_shared_mlp_backward(i.D, i.f, i.codes, i.scales, i.w_gu, i.w_down, i.dy, dx, dx, dwg, dwd)
    torch.cuda.synchronize()
    assert torch.equal(dx, want)


# ------------------------------------------------------------------ adapters

def _adapter_inputs(T, d, f, n, rank, dtype, ids, seed=0, scale=True):
    t = SimpleNamespace(T=T, d=d, f=f, n=n, dtype=dtype, D=S.desc(T, d, dtype), x=S.randn(seed, T, d, dtype=dtype),
                        w_gu=S.randn(seed + 1, 2 * f, d, scale=d ** -0.5, dtype=dtype),
                        w_down=S.randn(seed + 2, d, f, scale=f ** -0.5, dtype=dtype), y_in=S.randn(seed + 3, T, d),
                        ids=torch.as_tensor(ids, dtype=torch.int32).cuda())
    t.tables = [S.randn(seed + 4, n, 2 * rank, d, scale=d ** -0.5, dtype=dtype),
                S.randn(seed + 5, n, 2 * f, rank, scale=0.5 * rank ** -0.5, dtype=dtype),
                S.randn(seed + 6, n, rank, f, scale=f ** -0.5, dtype=dtype),
                S.randn(seed + 7, n, d, rank, scale=0.5 * rank ** -0.5, dtype=dtype),
                S.randn(seed + 8, n) if scale else None]
    return t


def _adapt(t, tables=None, y_in=True, x=None):
    ad = P.make_adapters(*(tables or t.tables))
    y, ws = Guarded((t.T, t.d), t.dtype), Guarded((P.omnimoe_shared_mlp_adapters_workspace_size(t.D, t.f, ad),), torch.uint8)
    ws.t.fill_(0xFF)
    P.omnimoe_shared_mlp_adapters(t.D, t.f, ad, t.x if x is None else x, t.w_gu, t.w_down, t.ids, t.y_in if y_in else None,
                                  y.t, ws=ws.t)
    torch.cuda.synchronize()
    y.check()
    ws.check()
    return y.t


def _adapt_reference(t, y_in=True):
    tables = list(t.tables)
    if tables[4] is None:
        tables[4] = torch.ones(t.n)
    y0 = t.y_in.to(F64) if y_in else torch.zeros((t.T, t.d), dtype=F64, device="cuda")
    return S.adapters_mlp(t.x.to(F64), t.w_gu.to(F64), t.w_down.to(F64), t.ids, tables, y0, t.dtype)


def _ids(kind, T, n, seed=0):
    g = torch.Generator().manual_seed(seed + 99)
    if kind == "none":
        return torch.full((T,), -1)
    if kind == "one":
        return torch.full((T,), n - 1)
    if kind == "own":
        return torch.arange(T) % n
    if kind == "runs":
        return torch.arange(T) * n // T
    ids = torch.randint(-1, n, (T,), generator=g)
    ids[torch.rand(T, generator=g) < 0.1] = 2 ** 31 - 1   # outside the table: no adapter
    ids[torch.rand(T, generator=g) < 0.05] = -(2 ** 31)
    ids[torch.rand(T, generator=g) < 0.05] = n
    return ids


ADAPT = [(1, 8, 8, 1, 8), (1, 64, 72, 3, 16), (2, 2048, 40, 5, 64), (15, 72, 64, 4, 24), (16, 64, 64, 16, 8),
         (17, 136, 264, 3, 16), (33, 520, 24, 40, 8), (48, 64, 64, 2, 256), (63, 40, 136, 64, 16), (64, 256, 256, 64, 32),
         (65, 64, 64, 7, 8), (66, 72, 520, 66, 24), (127, 264, 40, 5, 40), (128, 64, 128, 3, 256), (129, 520, 72, 129, 16),
         (300, 96, 200, 11, 48), (1000, 72, 136, 300, 8)]


@pytest.mark.parametrize("dtype", TYPES, ids=tid)
@pytest.mark.parametrize("kind", ["own", "mixed", "runs", "one", "none"])
@pytest.mark.parametrize("T,d,f,n,rank", ADAPT)
def test_adapters(T, d, f, n, rank, kind, dtype):
    print(f"[adapters] T={T} d={d} d_ff={f} n={n} rank={rank} {kind} {dtype}", file=sys.stderr, flush=True)
    t = _adapter_inputs(T, d, f, n, rank, dtype, _ids(kind, T, n), seed=T + d, scale=kind != "runs")
    y, bound = _adapt_reference(t)
    got = _adapt(t)
    within(got, y, bound, "y")
    assert torch.equal(got, _adapt(t)), "two runs differ"


@pytest.mark.parametrize("T,d,f,n,rank,kind", [(12288, 1024, 512, 9, 16, "mixed"), (12200, 1032, 1000, 40, 24, "runs"),
                                               (24576, 256, 136, 64, 8, "own"), (6144, 64, 1024, 3, 64, "mixed")])
def test_adapters_on_large_tiles(T, d, f, n, rank, kind):
    t = _adapter_inputs(T, d, f, n, rank, BF16, _ids(kind, T, n), seed=T)
    y, bound = _adapt_reference(t)
    got = _adapt(t)
    within(got, y, bound, "y")
    assert torch.equal(got, _adapt(t))


@pytest.mark.parametrize("dtype", TYPES, ids=tid)
@pytest.mark.parametrize("T", [20, 200])
def test_adapters_of_no_slots_and_without_y_in(T, dtype):
    t = _adapter_inputs(T, 72, 104, 4, 8, dtype, _ids("mixed", T, 4), seed=T)
    y, bound = _adapt_reference(t, y_in=False)
    within(_adapt(t, y_in=False), y, bound, "y without y_in")
    # no slots at all: the shared branch alone
    D, none = S.desc(T, 72, dtype), B.OmnimoeAdapters(n=0, rank=8)
    ws = torch.empty(P.omnimoe_shared_mlp_adapters_workspace_size(D, t.f, none), dtype=torch.uint8, device="cuda")
    out = torch.empty((T, 72), dtype=dtype, device="cuda")
    st = B.load_library().omnimoe_shared_mlp_adapters(
        B.ctypes.byref(D), t.f, B.ctypes.byref(none), B._ptr(t.x), B._ptr(t.w_gu), B._ptr(t.w_down), B._ptr(t.ids),
        B._ptr(t.y_in), B._ptr(out), B._ptr(ws), ws.numel(), B._stream(None))
    torch.cuda.synchronize()
    t.ids.fill_(-1)
    assert st == 0
    assert torch.equal(out, _adapt(t))


@pytest.mark.parametrize("T", [20, 200])
def test_adapters_of_a_descriptor_without_slots(T):
    # made directly, as a program without adapters has it
    t = _adapter_inputs(T, 72, 104, 4, 8, BF16, _ids("none", T, 4), seed=T)
    y = torch.empty((T, 72), dtype=BF16, device="cuda")
    P.omnimoe_shared_mlp_adapters(t.D, t.f, P.OmnimoeAdapters(n=0, rank=8), t.x, t.w_gu, t.w_down, t.ids, t.y_in, y)
    torch.cuda.synchronize()
    assert torch.equal(y, _adapt(t))


@pytest.mark.parametrize("dtype", TYPES, ids=tid)
@pytest.mark.parametrize("T", [20, 64, 65, 200, 700])
def test_a_slots_values_stay_with_its_tokens(T, dtype):
    # slot 2 holds NaN, slot 3 infinities, slot 5 is named by no token: the others' results are the same bits
    t = _adapter_inputs(T, 96, 72, 6, 16, dtype, _ids("own", T, 5), seed=T)
    clean = _adapt(t)
    bad = [v.clone() for v in t.tables]
    for v in bad[:4]:
        v[2], v[3], v[5] = float("nan"), float("inf"), float("nan")
    bad[4][5] = float("nan")
    got = _adapt(t, bad)
    kept = ((t.ids != 2) & (t.ids != 3))
    assert torch.equal(got[kept], clean[kept])
    assert not torch.isfinite(got[~kept].float()).any(1).all() and torch.isnan(got[t.ids == 2].float()).all()
    # and another token's x does not reach them either
    x = t.x.clone()
    x[0] = float("nan")
    got = _adapt(t, x=x)
    assert torch.equal(got[1:], clean[1:]) and torch.isnan(got[0].float()).all()


@pytest.mark.parametrize("dtype", TYPES, ids=tid)
@pytest.mark.parametrize("T", [20, 64, 65, 200, 700])
@pytest.mark.parametrize("table", range(4))
def test_a_slots_bad_values_reach_its_tokens(T, dtype, table):
    # an infinity in one row of one of slot 3's tables: every value that it enters is not finite. (The row of A: a rank-wide
    # value, and with it a column of B, all of the token's outputs. The row of B: a gate value, which silu and the down
    # projection spread, or one output.)
    t = _adapter_inputs(T, 96, 72, 6, 16, dtype, _ids("own", T, 5), seed=T)
    clean = _adapt(t)
    bad = [v.clone() for v in t.tables]
    bad[table][3, 7] = float("inf")
    got, mine = _adapt(t, bad), t.ids == 3
    assert mine.any() and torch.equal(got[~mine], clean[~mine])
    if table == 3:
        assert not torch.isfinite(got[mine][:, 7]).any()
        got[mine, 7] = clean[mine, 7]
        assert torch.equal(got, clean)
    else:
        assert not torch.isfinite(got[mine]).any()


def test_adapters_in_place_fp32_and_far_slots():
    t = _adapter_inputs(90, 64, 72, 5, 8, F32, _ids("mixed", 90, 5))
    want = _adapt(t)
    y, ad = t.y_in.clone(), P.make_adapters(*t.tables)
    P.omnimoe_shared_mlp_adapters(t.D, t.f, ad, t.x, t.w_gu, t.w_down, t.ids, y, y)
    torch.cuda.synchronize()
    assert torch.equal(y, want)
    # tables past 2^32 bytes: the last slot against the same slot in a small table
    n, rank, d, f = 8192, 128, 1040, 1040
    for T in (40, 100):
        s = _adapter_inputs(T, d, f, 1, rank, BF16, _ids("one", T, 1), seed=T)
        want = _adapt(s)
        big = [torch.zeros((n,) + v.shape[1:], dtype=v.dtype, device="cuda") for v in s.tables]
        for b, v in zip(big, s.tables):
            b[-1] = v[0]
        assert big[0].numel() * 2 > 2 ** 32 or big[1].numel() * 2 > 2 ** 32
        s.ids.fill_(n - 1)
        assert torch.equal(_adapt(s, big), want)
        del big


def test_adapters_in_several_passes():
    # more tokens than one pass takes (65536), the last pass short
    T, d, f, n = 65536 + 40, 32, 24, 3
    t = _adapter_inputs(T, d, f, n, 8, BF16, _ids("mixed", T, n), seed=3)
    y, bound = _adapt_reference(t)
    within(_adapt(t), y, bound, "y")


def test_adapters_whose_hidden_values_pass_4_gib():
    # [40000, 65536] bf16: 5.2e9 bytes, so that the last places' rows start beyond 2^32 of them
    T, d, f, n = 40000, 8, 65536, 2
    t = _adapter_inputs(T, d, f, n, 8, BF16, _ids("mixed", T, n), seed=5)
    got = _adapt(t)
    assert torch.isfinite(got).all()
    # tokens without a slot come last in the order of the slots; some from its start, its middle and its end
    order = torch.argsort(torch.where((t.ids < 0) | (t.ids >= n), n, t.ids), stable=True)
    some = torch.cat([order[:40], order[T // 2:T // 2 + 40], order[-80:]])
    y, bound = S.adapters_mlp(t.x[some].to(F64), t.w_gu.to(F64), t.w_down.to(F64), t.ids[some], t.tables,
                              t.y_in[some].to(F64), t.dtype)
    within(got[some], y, bound, "y")


# ------------------------------------------------------------------ the layer for a few tokens

def _few_inputs(T, d, nr, nc, dk, H, K, f, dtype, act="gelu", split=True, seed=0):
    w = d ** -0.5
    t = SimpleNamespace(T=T, d=d, H=H, K=K, f=f, dtype=dtype, act=act, split=split,
                        D=S.desc(T, d, dtype, n_rows=nr, n_cols=nc, d_key=dk, H=H, K=K, act=act,
                                 query_mode="split" if split else "shared"),
                        x=S.steps(seed, T, d, scale=1.0, step=1 / 16, dtype=dtype))
    step = 2.0 ** round(torch.log2(torch.tensor(w / 16)).item())
    t.kr = S.steps(seed + 1, H, nr, dk, scale=w, step=step, dtype=dtype)
    t.kc = S.steps(seed + 2, H, nc, dk, scale=w, step=step, dtype=dtype)
    t.u, t.v = S.randn(seed + 3, nr * nc, d, scale=w, dtype=dtype), S.randn(seed + 4, nr * nc, d, scale=w, dtype=dtype)
    t.w_gu = S.randn(seed + 5, 2 * f, d, scale=w, dtype=dtype) if f else None
    t.w_down = S.randn(seed + 6, d, f, scale=f ** -0.5, dtype=dtype) if f else None
    return t


def _few(t, outputs=True):
    y, idx, g = Guarded((t.T, t.d), F32), Guarded((t.T, t.H, t.K), torch.int32), Guarded((t.T, t.H, t.K), F32)
    ws = Guarded((P.omnimoe_layer_few_workspace_size(t.D, t.f),), torch.uint8)
    ws.t.fill_(0xFF)
    P.omnimoe_layer_forward_few(t.D, t.f, t.x, t.kr, t.kc, t.u, t.v, t.w_gu, t.w_down, y.t, idx.t if outputs else None,
                                g.t if outputs else None, ws=ws.t)
    torch.cuda.synchronize()
    for b in (y, idx, g, ws):
        b.check()
    return y.t, idx.t, g.t


FEW = [  # T, d, n_rows, n_cols, d_key, H, K, d_ff, act, split
    (1, 8, 1, 1, 8, 1, 1, 0, "gelu", False),
    (1, 16, 1, 5, 8, 2, 5, 8, "silu", True),
    (2, 64, 5, 1, 32, 3, 4, 40, "gelu", True),
    (3, 72, 7, 9, 72, 1, 63, 72, "gelu", False),        # K = N: every cell
    (5, 264, 16, 16, 128, 4, 16, 0, "silu", True),
    (7, 520, 120, 136, 264, 3, 13, 520, "silu", False),
    (8, 128, 64, 64, 64, 8, 64, 136, "gelu", True),
    (9, 512, 256, 256, 256, 4, 16, 512, "gelu", True),
    (13, 2048, 300, 257, 1024, 2, 33, 264, "gelu", True),
    (15, 96, 513, 17, 40, 2, 32, 2048, "silu", True),
    (16, 1024, 320, 320, 512, 1, 64, 1024, "gelu", True),
    (16, 256, 1024, 3, 128, 5, 8, 64, "gelu", True),
    (4, 64, 2500, 3, 32, 1, 16, 64, "gelu", True),
    (2, 64, 3, 4096, 32, 2, 64, 8, "gelu", True),
    (1, 4096, 64, 64, 2048, 2, 16, 4096, "gelu", True),
    (16, 3200, 33, 40, 1600, 17, 7, 24, "silu", True),
]


@pytest.mark.parametrize("dtype", TYPES, ids=tid)
@pytest.mark.parametrize("case", FEW, ids=lambda c: "-".join(map(str, c)))
def test_few(case, dtype):
    print(f"[few] {case} {dtype}", file=sys.stderr, flush=True)
    T, d, nr, nc, dk, H, K, f, act, split = case
    t = _few_inputs(T, d, nr, nc, dk, H, K, f, dtype, act, split, seed=T + d)
    idx, gates, y, bound = S.few_layer(t.x, t.kr, t.kc, t.u, t.v, t.w_gu, t.w_down, K, act, split)
    gy, gi, gg = _few(t)
    assert torch.equal(gi.long(), idx), "selection"
    # scores are exact sums of exact logits; exp and the division in fp32, the K terms' sum
    within(gg, gates, (K + 16) * S.U32 * gates + 1e-30, "gates")
    within(gy, y, bound, "y")
    again = _few(t)
    assert torch.equal(gy, again[0]) and torch.equal(gg, again[2])
    assert torch.equal(_few(t, outputs=False)[0], gy)


def test_few_wide_bf16():
    t = _few_inputs(3, 8192, 24, 24, 4096, 2, 20, 8192, BF16, seed=1)
    idx, gates, y, bound = S.few_layer(t.x, t.kr, t.kc, t.u, t.v, t.w_gu, t.w_down, t.K, "gelu", True)
    gy, gi, gg = _few(t)
    assert torch.equal(gi.long(), idx)
    within(gy, y, bound, "y")


@pytest.mark.parametrize("nr,nc,K", [(16, 16, 16), (100, 300, 64), (1024, 1024, 64), (4096, 2, 64)])
def test_few_ties(nr, nc, K):
    # x = 0: every score is equal, the lowest ids win with equal gates, and y is zero; then few distinct logits
    t = _few_inputs(2, 64, nr, nc, 32, 2, K, 64, BF16, seed=nr)
    t.x.zero_()
    y, idx, g = _few(t)
    assert not y.any() and torch.equal(idx, torch.arange(K, device="cuda", dtype=torch.int32).expand(2, 2, K))
    assert torch.allclose(g, torch.full_like(g, 1 / K), rtol=1e-6, atol=0)
    t.x[:, 0] = 1.0
    t.kr.copy_(torch.sign(t.kr))
    t.kc.copy_(torch.sign(t.kc))
    want = S.few_layer(t.x, t.kr, t.kc, t.u, t.v, t.w_gu, t.w_down, K, "gelu", True)
    y, idx, g = _few(t)
    assert torch.equal(idx.long(), want[0])
    within(y, want[2], want[3], "y")


def test_few_agrees_with_the_layer():
    t = _few_inputs(11, 512, 256, 256, 256, 4, 16, 512, BF16, seed=4)
    y, idx, g = _few(t)
    ly, li, lg = torch.empty_like(y), torch.empty_like(idx), torch.empty_like(g)
    P.omnimoe_layer_forward(t.D, t.x, t.kr, t.kc, t.u, t.v, ly, li, lg)
    routed = ly.clone()
    P.omnimoe_shared_mlp(t.D, t.f, t.x, t.w_gu, t.w_down, ly)
    assert torch.equal(idx, li)
    # gates: both within K + 16 units of the exact ones; y: the layer's shared branch rounds its hidden values to bf16
    assert ((g - lg).abs() <= 2 * (t.K + 16) * S.U32 * lg).all()
    a = t.x.to(F64) @ t.w_gu.to(F64).t()
    a = (S.silu(a[:, :t.f]) * a[:, t.f:]).abs()
    _, _, _, bound = S.few_layer(t.x, t.kr, t.kc, t.u, t.v, t.w_gu, t.w_down, t.K, "gelu", True)
    within(y, ly.to(F64), 2 * bound + 2.0 ** -8 * (a @ t.w_down.to(F64).abs().t()), "y")
    t.f, t.w_gu, t.w_down = 0, None, None
    within(_few(t)[0], routed.to(F64), 2 * bound, "routed")


def _same_or_within(got, want, bound, what):
    """Infinities and NaN where the 64-bit form has them, the other values within their bound."""
    fine = torch.isfinite(want)
    assert _same(torch.where(fine, 0.0, got.to(F64)), torch.where(fine, 0.0, want)), what
    within(torch.where(fine, got.to(F64), 0.0), torch.where(fine, want, 0.0), torch.where(fine, bound, 0.0), what)


@pytest.mark.parametrize("dtype", TYPES, ids=tid)
@pytest.mark.parametrize("d", [8, 520, 1544, 2056])
def test_few_infinity_at_the_end_of_a_u_row(d, dtype):
    # one expert of a token's picks has an infinite last value in its u row, whose x there is 1: its h is an infinity, and
    # so is y (GELU of it, times nonzero gates and v values of either sign). No row of a wave's loads ends with the row.
    t = _few_inputs(2, d, 16, 16, 8, 2, 5, 0, dtype, split=False, seed=d)
    t.x[:, -1] = 1.0
    t.v.copy_(torch.where(t.v == 0, 1.0, t.v))
    y, idx, _ = _few(t)
    t.u[idx[0, 1, 3].long(), -1] = float("inf")
    want = S.few_layer(t.x, t.kr, t.kc, t.u, t.v, None, None, t.K, "gelu", False)
    assert torch.isinf(want[2][0]).all()
    y, idx, _ = _few(t)
    assert torch.equal(idx.long(), want[0])
    _same_or_within(y, want[2], want[3], "y")


@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("dtype", TYPES, ids=tid)
def test_few_hidden_values_at_the_end_of_the_range(dtype, sign):
    # token 0: a = 2^140, an infinity in fp32, as y is then; token 1: a = 2^128 - 2^116, which fp32 holds and which lies past
    # bf16's largest value; token 2: neither
    t = _few_inputs(3, 64, 16, 16, 32, 2, 4, 40, dtype, seed=11)
    t.x[:, 60:] = 0
    t.x[0, 60] = t.x[1, 61] = t.x[1, 62] = 1.0
    t.w_gu[:, 60:] = 0
    t.w_gu[0, 60], t.w_gu[40, 60] = 2.0 ** 70, sign * 2.0 ** 70
    t.w_gu[1, 61], t.w_gu[41, 61], t.w_gu[41, 62] = 2.0 ** 64, sign * 2.0 ** 64, sign * -(2.0 ** 52)
    t.w_down[:, 0] = torch.where(t.w_down[:, 0] == 0, 1.0, t.w_down[:, 0])
    t.w_down[:, 1] *= 2.0 ** -10
    want = S.few_layer(t.x, t.kr, t.kc, t.u, t.v, t.w_gu, t.w_down, t.K, "gelu", True)
    y, idx, _ = _few(t)
    assert torch.equal(idx.long(), want[0])
    most = want[2].to(F32).to(F64)  # 2^140 w: an infinity
    assert torch.isinf(most[0]).all() and torch.isfinite(most[1:]).all()
    _same_or_within(y, most, want[3] + 2 * S.U32 * want[2].abs(), "y")


@pytest.mark.parametrize("dtype", TYPES, ids=tid)
@pytest.mark.parametrize("T,d,f", [(1, 64, 8), (5, 136, 136), (16, 64, 1032)])
def test_few_infinite_weights_of_the_down_projection(T, d, f, dtype):
    # columns 3 and 20 of the output have one infinite weight each, column 33 two of either sign: infinities of the hidden
    # values' signs, and NaN where the two meet; a hidden value of zero gives NaN too
    t = _few_inputs(T, d, 16, 16, 32, 2, 4, f, dtype, seed=f)
    t.w_down[3, f - 1], t.w_down[20, 0] = float("inf"), -float("inf")
    t.w_down[33, 1], t.w_down[33, f - 2] = float("inf"), -float("inf")
    t.w_gu[f] = 0  # feature 0's hidden value
    want = S.few_layer(t.x, t.kr, t.kc, t.u, t.v, t.w_gu, t.w_down, t.K, "gelu", True)
    assert torch.isinf(want[2][:, 3]).all() and torch.isnan(want[2][:, 20]).all() and not torch.isfinite(want[2][:, 33]).any()
    y, idx, _ = _few(t)
    assert torch.equal(idx.long(), want[0])
    _same_or_within(y, want[2], want[3], "y")


@pytest.mark.parametrize("K", [4, 16, 64])
@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")], ids=["inf", "-inf", "nan"])
@pytest.mark.parametrize("dtype", TYPES, ids=tid)
def test_few_selects_as_the_layer_where_keys_are_not_finite(dtype, value, K):
    t = _few_inputs(4, 256, 64, 64, 128, 2, K, 0, dtype, seed=6)
    t.x[:, 0] = t.x[:, 128] = 1.0
    t.kr[:, 3::7, 0] = value
    t.kc[:, 5::9, 0] = value
    y, idx, g = _few(t)
    ly, li, lg = torch.empty_like(y), torch.empty_like(idx), torch.empty_like(g)
    P.omnimoe_layer_forward(t.D, t.x, t.kr, t.kc, t.u, t.v, ly, li, lg)
    torch.cuda.synchronize()
    assert torch.equal(idx, li)
    # both within K + 16 units of the exact gates; NaN in the same places
    assert torch.equal(torch.isnan(g), torch.isnan(lg)) and torch.equal(torch.isnan(y), torch.isnan(ly))
    assert (torch.nan_to_num(g - lg).abs() <= 2 * (K + 16) * S.U32 * torch.nan_to_num(lg)).all()


# ------------------------------------------------------------------ graphs, streams, together


@pytest.mark.parametrize("dtype,d,f", [(BF16, 8, 65536), (BF16, 8192, 72), (F32, 8, 65536), (F32, 4096, 72)],
                         ids=lambda v: tid(v) if v in TYPES else str(v))
def test_largest_widths(dtype, d, f):
    i = _backward_inputs(3, d, f, dtype, seed=3)
    want, bound = S.mlp_backward_bounds(S.dequantise(i.codes, i.scales), i.w_gu.to(F64), i.w_down.to(F64), i.dy.to(F64),
                                        i.dx_in.to(F64), dtype)
    for g, w, b, name in zip(_backward(i), want, bound, ("dx", "dw_gu", "dw_down")):
        within(g, w, b, name)
    for T in (3, 40, 70):
        t = _adapter_inputs(T, d, f, 3, 16, dtype, _ids("mixed", T, 3), seed=4)
        y, bound = _adapt_reference(t)
        within(_adapt(t), y, bound, f"adapters, {T} tokens")
    t = _few_inputs(3, d, 16, 16, 8, 2, 5, f, dtype, split=False, seed=5)
    want = S.few_layer(t.x, t.kr, t.kc, t.u, t.v, t.w_gu, t.w_down, t.K, "gelu", False)
    y, idx, _ = _few(t)
    assert torch.equal(idx.long(), want[0])
    within(y, want[2], want[3], "few")

def _calls(seed=0, T=40):
    """One call of each operator on buffers of its own: (name, call, outputs, workspace)."""
    b = _backward_inputs(T, 128, 72, BF16, seed)
    bo = [torch.zeros((T, 128), dtype=BF16, device="cuda"), torch.zeros_like(b.w_gu), torch.zeros_like(b.w_down)]
    bw = torch.zeros(P.omnimoe_shared_mlp_backward_workspace_size(b.D, b.f), dtype=torch.uint8, device="cuda")
    out = [("backward", lambda s=None: P.omnimoe_shared_mlp_backward(
        b.D, b.f, b.codes, b.scales, b.w_gu, b.w_down, b.dy, b.dx_in, *bo, ws=bw, stream=s), bo, bw)]
    for T2 in (T, 3 * T):
        a = _adapter_inputs(T2, 64, 72, 5, 16, BF16, _ids("mixed", T2, 5), seed + 1)
        ad = P.make_adapters(*a.tables)
        ay = torch.zeros((T2, 64), dtype=BF16, device="cuda")
        aw = torch.zeros(P.omnimoe_shared_mlp_adapters_workspace_size(a.D, a.f, ad), dtype=torch.uint8, device="cuda")
        out.append((f"adapters {T2}", lambda s=None, a=a, ad=ad, ay=ay, aw=aw: P.omnimoe_shared_mlp_adapters(
            a.D, a.f, ad, a.x, a.w_gu, a.w_down, a.ids, a.y_in, ay, ws=aw, stream=s), [ay], aw))
    f = _few_inputs(9, 256, 64, 64, 128, 4, 16, 136, BF16, seed=seed + 2)
    fy, fi = torch.zeros((9, 256), dtype=F32, device="cuda"), torch.zeros((9, 4, 16), dtype=torch.int32, device="cuda")
    fw = torch.zeros(P.omnimoe_layer_few_workspace_size(f.D, f.f), dtype=torch.uint8, device="cuda")
    out.append(("few", lambda s=None: P.omnimoe_layer_forward_few(f.D, f.f, f.x, f.kr, f.kc, f.u, f.v, f.w_gu, f.w_down, fy,
                                                                  fi, None, ws=fw, stream=s), [fy, fi], fw))
    c = S.randn(seed + 9, T, 96, dtype=BF16)
    D = S.desc(T, 96, BF16)
    co = [torch.zeros((T, 96), dtype=torch.uint8, device="cuda"), torch.zeros((T, 3), dtype=torch.uint8, device="cuda"),
          torch.zeros((T, 96), dtype=BF16, device="cuda")]

    def checkpoint(s=None):
        P.omnimoe_checkpoint_store(D, c, co[0], co[1], stream=s)
        P.omnimoe_checkpoint_load(D, co[0], co[1], co[2], stream=s)
    out.append(("checkpoint", checkpoint, co, torch.zeros(256, dtype=torch.uint8, device="cuda")))
    return out


def test_graph_replays():
    for name, call, outs, ws in _calls():
        call()
        torch.cuda.synchronize()
        want = [o.clone() for o in outs]
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            call()
        for k in range(4):
            for o in outs:
                o.fill_(k)
            ws.fill_(0xFF - k)  # eager work between the replays
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want)), f"{name}, replay {k}"


def test_two_graphs_share_a_workspace():
    # replayed one after the other on one stream
    one, two = _calls(0), _calls(7)
    for (name, a, ao, aw), (_, b, bo, _) in zip(one, two):
        a()
        b()
        torch.cuda.synchronize()
        want = [o.clone() for o in ao]
        s = torch.cuda.Stream()
        graphs = []
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                a()
            graphs.append(g)
        for _ in range(3):
            for o in ao:
                o.zero_()
            for g in graphs:
                g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(ao, want)), name


def test_graphs_of_different_calls_share_a_workspace():
    # one workspace under the graphs of all operators, each of two sets of inputs, replayed in turn and in the other order
    ws = torch.zeros(1 << 22, dtype=torch.uint8, device="cuda")
    calls = []
    for T, seed in ((40, 0), (97, 7)):
        b = _backward_inputs(T, 128, 72, BF16, seed)
        assert P.omnimoe_shared_mlp_backward_workspace_size(b.D, b.f) <= ws.numel()
        outs = [torch.zeros((T, 128), dtype=BF16, device="cuda"), torch.zeros_like(b.w_gu), torch.zeros_like(b.w_down)]
        calls.append((f"backward {T}", outs, lambda b=b, o=outs: P.omnimoe_shared_mlp_backward(
            b.D, b.f, b.codes, b.scales, b.w_gu, b.w_down, b.dy, b.dx_in, *o, ws=ws)))
        a = _adapter_inputs(T, 64, 72, 5, 16, BF16, _ids("mixed", T, 5), seed + 1)
        ad = P.make_adapters(*a.tables)
        assert P.omnimoe_shared_mlp_adapters_workspace_size(a.D, a.f, ad) <= ws.numel()
        outs = [torch.zeros((T, 64), dtype=BF16, device="cuda")]
        calls.append((f"adapters {T}", outs, lambda a=a, ad=ad, o=outs: P.omnimoe_shared_mlp_adapters(
            a.D, a.f, ad, a.x, a.w_gu, a.w_down, a.ids, a.y_in, *o, ws=ws)))
        f = _few_inputs(3 + seed, 256, 64, 64, 128, 4, 16, 136, BF16, seed=seed + 2)
        assert P.omnimoe_layer_few_workspace_size(f.D, f.f) <= ws.numel()
        outs = [torch.zeros((f.T, 256), dtype=F32, device="cuda"), torch.zeros((f.T, 4, 16), dtype=torch.int32, device="cuda")]
        calls.append((f"few {f.T}", outs, lambda f=f, o=outs: P.omnimoe_layer_forward_few(
            f.D, f.f, f.x, f.kr, f.kc, f.u, f.v, f.w_gu, f.w_down, *o, None, ws=ws)))
    want, graphs, s = [], [], torch.cuda.Stream()
    for _, outs, call in calls:
        call()
        torch.cuda.synchronize()
        want.append([o.clone() for o in outs])
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            call()
        graphs.append(graph)
    for order in (graphs, graphs[::-1], graphs[::2] + graphs[1::2]):
        for _, outs, _ in calls:
            for o in outs:
                o.zero_()
        for graph in order:
            graph.replay()
        torch.cuda.synchronize()
        for (name, outs, _), w in zip(calls, want):
            assert all(torch.equal(x, y) for x, y in zip(outs, w)), name


def test_calls_on_two_streams():
    one, two = _calls(0), _calls(7)
    for _, call, _, _ in one + two:
        call()
    torch.cuda.synchronize()
    want = [[o.clone() for o in outs] for _, _, outs, _ in one + two]
    for _, _, outs, _ in one + two:
        for o in outs:
            o.zero_()
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        for (_, a, _, _), (_, b, _, _) in zip(one, two):
            a(s1)
            b(s2)
    torch.cuda.synchronize()
    for (name, _, outs, _), w in zip(one + two, want):
        assert all(torch.equal(x, y) for x, y in zip(outs, w)), name


def test_workspaces_belong_to_the_calls_stream(monkeypatch):
    # a call that makes its own workspace takes it from the pool of the stream it runs on
    b, s = _backward_inputs(65, 64, 72, BF16), torch.cuda.Stream()
    want = _backward(b)
    outs = [torch.empty_like(o) for o in want]
    made, empty = [], torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **k: made.append(torch.cuda.current_stream()) or empty(*a, **k))
    s.wait_stream(torch.cuda.current_stream())
    P.omnimoe_shared_mlp_backward(b.D, b.f, b.codes, b.scales, b.w_gu, b.w_down, b.dy, b.dx_in, *outs, stream=s)
    torch.cuda.synchronize()
    assert made == [s]
    assert all(torch.equal(o, w) for o, w in zip(outs, want))


@pytest.mark.parametrize("dtype", TYPES, ids=tid)
def test_training_step_with_the_routed_layer(dtype):
    """Forward: the routed layer, the shared branch, the checkpoint of x. Way back: x from the checkpoint, then the expert,
    router and shared gradients, whose dx is one sum. (x holds values that the checkpoint keeps, so that the gates of the
    forward pass and the x of the way back belong together.)"""
    T, d, f = 300, 128, 136
    w = d ** -0.5
    D = S.desc(T, d, dtype, n_rows=16, n_cols=16, d_key=64, H=2, K=4)
    x = S.quantise(S.randn(1, T, d, dtype=dtype))[0].to(dtype)
    kr, kc = S.randn(2, 2, 16, 64, scale=w, dtype=dtype), S.randn(3, 2, 16, 64, scale=w, dtype=dtype)
    u, v = S.randn(4, 256, d, scale=w, dtype=dtype), S.randn(5, 256, d, scale=w, dtype=dtype)
    wg, wd = S.randn(6, 2 * f, d, scale=w, dtype=dtype), S.randn(7, d, f, scale=f ** -0.5, dtype=dtype)
    f32 = lambda *s: torch.zeros(s, dtype=F32, device="cuda")  # noqa: E731
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    y, idx, gates = f32(T, d), i32(T, 2, 4), f32(T, 2, 4)
    P.omnimoe_layer_forward(D, x, kr, kc, u, v, y, idx, gates)
    P.omnimoe_shared_mlp(D, f, x, wg, wd, y)
    codes, scales = torch.zeros((T, d), dtype=torch.uint8, device="cuda"), torch.zeros((T, d // 32), dtype=torch.uint8, device="cuda")
    P.omnimoe_checkpoint_store(D, x, codes, scales)
    kept = torch.empty_like(x)
    P.omnimoe_checkpoint_load(D, codes, scales, kept)
    assert torch.equal(kept, x)
    dy = S.randn(8, T, d)
    M = T * 8
    perm, active, off, na = i32(M), i32(256), i32(257), i32(1)
    P.omnimoe_schedule(D, idx, perm, active, off, na)
    dx, du, dv, dg, ds = f32(T, d), f32(256, d), f32(256, d), f32(T, 2, 4), f32(T, 2, 4)
    P.omnimoe_expert_backward(D, kept, u, v, idx, gates, perm, off, na, dy, dx, du, dv, dg, ds)
    P.omnimoe_route_backward(D, kept, kr, kc, idx, ds, dx, f32(2, 16, 64), f32(2, 16, 64))
    out, dwg, dwd = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wd)
    P.omnimoe_shared_mlp_backward(D, f, codes, scales, wg, wd, dy, dx, out, dwg, dwd)
    X = kept.to(F64)
    want, bound = S.mlp_backward_bounds(X, wg.to(F64), wd.to(F64), dy.to(F64), dx.to(F64), dtype)
    for g, r, b, name in zip((out, dwg, dwd), want, bound, ("dx", "dw_gu", "dw_down")):
        within(g, r, b, name)
    # dx against differences of the whole layer's loss on the routing of the forward pass (its scores' softmax included)
    to = S.randn(9, T, d).to(F64)
    e = idx.long().flatten(1)
    i, j = idx.long() // 16, idx.long() % 16
    U, V = u.to(F64)[e], v.to(F64)[e]
    h_ = torch.arange(2, device="cuda").view(1, 2, 1).expand_as(i)

    def loss(z):
        s = (kr.to(F64)[h_, i] * z[:, None, None, :64]).sum(-1) + (kc.to(F64)[h_, j] * z[:, None, None, 64:]).sum(-1)
        g = torch.softmax(s, -1).flatten(1)
        a = torch.matmul(U, z[:, :, None])[:, :, 0]
        r = ((g * 0.5 * a * torch.erfc(-a * 0.5 ** 0.5))[:, None] @ V)[:, 0]
        q = z @ wg.to(F64).t()
        return float((dy.to(F64) * (r + (S.silu(q[:, :f]) * q[:, f:]) @ wd.to(F64).t())).sum())

    h = 1e-5
    slope = (loss(X + h * to) - loss(X - h * to)) / (2 * h)
    mine = float((out.to(F64) * to).sum())
    # the shared share's and the rounding's bound along the direction; the routed share is fp32 (its sums of eight tasks and
    # 128 products are within 1e-4 of their terms); the difference's own error
    routed = float((dx.abs().to(F64) * to.abs()).sum())
    assert abs(slope - mine) <= float((bound[0] * to.abs()).sum()) + 1e-4 * routed + 1e-6 * (1 + abs(slope))


def test_decode_step_with_adapters():
    """A decode step: the routed branch for a few tokens, then the shared branch with each request's adapter on top."""
    t = _few_inputs(12, 256, 64, 64, 128, 4, 16, 0, BF16, seed=3)
    y, idx, _ = _few(t)
    a = _adapter_inputs(12, 256, 136, 4, 16, BF16, _ids("own", 12, 4), seed=6)
    a.x, a.y_in, a.D = t.x, y, t.D
    out, bound = _adapt_reference(a)
    within(_adapt(a), out, bound, "y")
    # without adapters it is the whole layer of the few-token call, but for the hidden values' rounding to bf16
    a.ids.fill_(-1)
    plain = _adapt(a)
    t.f, t.w_gu, t.w_down = a.f, a.w_gu, a.w_down
    whole, _, _ = _few(t)
    out, bound = _adapt_reference(a)
    within(plain, whole.to(F64), 2 * bound, "without adapters")
