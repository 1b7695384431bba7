"""The operators of include/omnimoe_block.h on the CPU: what the library exports, the refusals of every entry point (which
come from the host-side checks, before anything is launched), and the plain 64-bit forms that the GPU tests compare with."""
import ctypes
import os
import re

import pytest
import torch

import block_support as K
import ffn_support as S
import paper_2602_05711_amd as P
from paper_2602_05711_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED, ALIGN, WORKSPACE = 0, 1, 2, 3, 4
A = ctypes.c_void_p(0x10000)  # aligned, never dereferenced: the checks fail first
BAD = ctypes.c_void_p(0x10004)
BIG = ctypes.c_size_t(1 << 40)


def _lib():
    return P.load_library()


def _desc(T=100, d=64, dtype=torch.bfloat16, **kw):
    return S.desc(T, d, dtype, **kw)


def _header():
    with open(os.path.join(ROOT, "include", "omnimoe_block.h")) as f:
        return f.read()


def test_header_matches_exports():
    names = sorted(set(re.findall(r"^omnimoe_status\s+(omnimoe_\w+)\(", _header(), flags=re.M)))
    assert sorted(P.EXPORTED_BLOCK) == names
    for n in names:
        assert hasattr(_lib(), n) and hasattr(P, n)


def test_orders_and_product_layout():
    assert ctypes.sizeof(B.OmnimoeProduct) == 20 and B.OmnimoeProduct.y_order.offset == 16
    for name, value in P.ORDERS.items():
        assert re.search(rf"OMNIMOE_ORDER_{name.upper()} = {value}\b", _header())


# ------------------------------------------------------------------ the joint

def _join(desc, change=(), eps=1e-6, gate_width=1):
    args = [A] * 8  # x, y, gate, w_out, scale, w_in, x_out, n
    for i, v in change:
        args[i] = v
    return _lib().omnimoe_block_join(ctypes.byref(desc), eps, gate_width, *args, None)


def test_join_refusals():
    d = _desc()
    for i in (0, 1, 2, 6, 7):
        change = [(i, None)] + ([(5, None)] if i == 1 else [])
        assert _join(d, change) == INVALID, i
    for i in range(8):
        assert _join(d, [(i, BAD)]) == ALIGN, i
    for eps in (0.0, 1e-31, -1e-6, float("inf"), float("nan")):
        assert _join(d, eps=eps) == INVALID
    for width in (-1, 2, 63, 65):
        assert _join(d, gate_width=width) == INVALID
    assert _join(_desc(d=60)) == INVALID and _join(_desc(T=-1)) == INVALID
    assert _join(_desc(T=0), [(i, None) for i in (0, 2, 6, 7)]) == OK
    assert _lib().omnimoe_block_join(None, 1e-6, 0, *[A] * 8, None) == INVALID


def _join_back(desc, change=(), eps=1e-6, gate_width=1, ws=BIG):
    # x_out, y, gate, w_out, scale, w_in, dx_out, dn, dx, dy, dgate, dw_out, dscale, dw_in, workspace
    args = [A] * 15
    for i, v in change:
        args[i] = v
    return _lib().omnimoe_block_join_backward(ctypes.byref(desc), eps, gate_width, *args, ws, None)


def test_join_backward_refusals():
    d = _desc()
    for i in (0, 2, 7, 8, 9, 10, 11, 12, 13, 14):
        assert _join_back(d, [(i, None)]) == INVALID, i
    for i in range(15):
        assert _join_back(d, [(i, BAD)]) == ALIGN, i
    assert _join_back(d, [(1, None), (5, None)]) == INVALID  # nothing to do
    assert _join_back(d, [(5, None), (6, None)]) == INVALID  # no gradient comes in
    assert _join_back(d, ws=ctypes.c_size_t(16)) == WORKSPACE
    assert _join_back(d, eps=0.0) == INVALID and _join_back(d, gate_width=7) == INVALID
    # what an absent input makes unneeded is not asked for
    assert _join_back(d, [(i, None) for i in (1, 2, 3, 4, 9, 10, 11, 12)], ws=ctypes.c_size_t(16)) == WORKSPACE
    assert _join_back(d, [(i, None) for i in (0, 5, 7, 13)], ws=ctypes.c_size_t(16)) == WORKSPACE
    assert _join_back(_desc(T=0), [(i, None) for i in range(15)]) == OK
    assert _join_back(_desc(T=0), [(13, BAD)]) == ALIGN
    n = ctypes.c_size_t(0)
    size = _lib().omnimoe_block_join_backward_workspace_size
    assert size(ctypes.byref(d), None) == INVALID and size(None, ctypes.byref(n)) == INVALID
    assert size(ctypes.byref(d), ctypes.byref(n)) == OK and n.value >= 2 * 64 * 4


# ------------------------------------------------------------------ products

def _q(n_in=64, n_out=64, swiglu=0, x_order=1, y_order=1):
    return B.OmnimoeProduct(n_in=n_in, n_out=n_out, swiglu=swiglu, x_order=x_order, y_order=y_order)


CALLS = {  # entry point: its pointers, and which of them must be there
    "omnimoe_grouped_product": 5,     # x, w, offsets, perm, y
    "omnimoe_grouped_product_dx": 5,  # dy, w, offsets, perm, dx
    "omnimoe_grouped_product4": 6,    # x, codes, scales, offsets, perm, y
}


def _product(fn, desc, q, change=()):
    args = [A] * CALLS[fn]
    for i, v in change:
        args[i] = v
    return getattr(_lib(), fn)(ctypes.byref(desc), None if q is None else ctypes.byref(q), *args, None)


@pytest.mark.parametrize("fn", sorted(CALLS))
def test_product_refusals(fn):
    d = _desc(K=2)
    for i in range(CALLS[fn]):
        assert _product(fn, d, _q(), [(i, None)]) == INVALID, i
        assert _product(fn, d, _q(), [(i, BAD)]) == ALIGN, i
    assert _product(fn, d, None) == INVALID
    for bad in (dict(n_in=0), dict(n_in=12), dict(n_out=-8), dict(n_out=65544), dict(swiglu=2), dict(x_order=3),
                dict(x_order=-1), dict(y_order=2), dict(y_order=-1)):
        assert _product(fn, d, _q(**bad)) == INVALID, bad
    assert _product(fn, _desc(n_rows=64, n_cols=65), _q()) == UNSUPPORTED
    assert _product(fn, d, _q(n_in=65536, n_out=32768)) == UNSUPPORTED  # 4 GiB
    assert _product(fn, _desc(dtype=torch.float32), _q(n_in=32768, n_out=32768)) == UNSUPPORTED
    # 2^31 - 4 tasks
    assert _product(fn, _desc(T=2304167, H=233, K=4, n_rows=2, n_cols=2, query_mode="shared"), _q()) == UNSUPPORTED
    assert _product(fn, _desc(T=0), _q(), [(i, None) for i in range(CALLS[fn])]) == OK
    assert _product(fn, _desc(d=60), _q()) == INVALID
    if fn.endswith("dx"):
        assert _product(fn, d, _q(swiglu=1)) == INVALID and _product(fn, d, _q(x_order=2)) == INVALID
    if fn.endswith("4"):
        assert _product(fn, d, _q(n_in=72)) == INVALID  # blocks of 32


def _dw(desc, q, change=(), ws=BIG):
    args = [A] * 6  # x, dy, offsets, perm, dw, workspace
    for i, v in change:
        args[i] = v
    return _lib().omnimoe_grouped_product_dw(ctypes.byref(desc), ctypes.byref(q), *args, ws, None)


def test_product_dw_refusals():
    d = _desc(T=6000, n_rows=1, n_cols=1)  # one expert: parts in the workspace
    for i in (0, 1, 3, 4, 5):
        assert _dw(d, _q(), [(i, None)]) == INVALID, i
    for i in range(6):
        assert _dw(d, _q(), [(i, BAD)]) == ALIGN, i
    assert _dw(_desc(), _q(), [(2, None)]) == INVALID
    assert _dw(d, _q(), ws=ctypes.c_size_t(16)) == WORKSPACE
    assert _dw(d, _q(swiglu=1)) == INVALID
    size, n = _lib().omnimoe_grouped_product_dw_workspace_size, ctypes.c_size_t(0)
    assert size(ctypes.byref(d), ctypes.byref(_q()), ctypes.byref(n)) == OK
    assert n.value >= 2 * 64 * 64 * 4 and n.value % (64 * 64 * 4) == 0
    assert size(ctypes.byref(d), ctypes.byref(_q()), None) == INVALID
    assert size(ctypes.byref(d), None, ctypes.byref(n)) == INVALID
    assert size(ctypes.byref(d), ctypes.byref(_q(swiglu=1)), ctypes.byref(n)) == INVALID
    assert size(ctypes.byref(_desc(n_rows=32, n_cols=32)), ctypes.byref(_q()), ctypes.byref(n)) == OK and n.value == 0


@pytest.mark.parametrize("rows,experts,n_in,n_out,parts", [(65536, 4, 1024, 1024, 8), (32768, 1, 4096, 4096, 2),
                                                           (16384, 1, 2048, 2048, 8), (65536, 16, 1024, 2048, 1)])
def test_product_dw_parts(rows, experts, n_in, n_out, parts):
    # long sums of few experts: tiles of 256 (0.64 to 0.98 of the time that those of 128 take), as many parts as fill 512 tiles
    d = _desc(T=rows, n_rows=1, n_cols=experts, dtype=torch.bfloat16, query_mode="shared")
    size, n = _lib().omnimoe_grouped_product_dw_workspace_size, ctypes.c_size_t(0)
    assert size(ctypes.byref(d), ctypes.byref(_q(n_in=n_in, n_out=n_out)), ctypes.byref(n)) == OK
    assert n.value == (parts * experts * n_in * n_out * 4 if parts > 1 else 0)


@pytest.mark.parametrize("fn", ["omnimoe_weights4_store", "omnimoe_weights4_load"])
def test_weights4_refusals(fn):
    call = getattr(_lib(), fn)
    d = _desc()
    for i in range(3):
        for v, status in ((None, INVALID), (BAD, ALIGN)):
            args = [A] * 3
            args[i] = v
            assert call(ctypes.byref(d), ctypes.byref(_q()), *args, None) == status
    assert call(ctypes.byref(d), ctypes.byref(_q(n_in=72)), A, A, A, None) == INVALID
    assert call(ctypes.byref(_desc(n_rows=64, n_cols=65)), ctypes.byref(_q()), A, A, A, None) == UNSUPPORTED


def test_binding_refuses_before_the_call():
    bf = torch.bfloat16
    d = _desc(T=4)
    x, y, w = torch.zeros(4, 64, dtype=bf), torch.zeros(4, 64), torch.zeros(64)
    with pytest.raises(ValueError, match="not on a GPU"):
        P.omnimoe_block_join(d, 1e-6, x, y, None, w, None, w, x, x)
    with pytest.raises(ValueError, match="gate must be contiguous"):  # (a gate of the wrong size, on the same device)
        B._ffn_refuse("omnimoe_block_join", 0, "gate", torch.zeros(5, 1, dtype=bf), bf, 4)
    with pytest.raises(ValueError, match="x is torch.float32"):
        P.omnimoe_block_join(d, 1e-6, y, y, None, w, None, w, x, x)
    with pytest.raises(ValueError, match="not on a GPU"):
        P.omnimoe_grouped_product(d, P.make_product(64, 64), x, torch.zeros(256, 64, 64, dtype=bf), None, None, x)
    q = P.make_product(64, 32, swiglu=True, x_order="token")
    assert (q.n_in, q.n_out, q.swiglu, q.x_order, q.y_order) == (64, 32, 1, 2, 0)
    with pytest.raises(KeyError):
        P.make_product(64, 32, x_order="expert")


def test_heads_times_experts_past_32_bits_without_tokens():
    # no tokens: nothing is divided by H K, which has no 32-bit value here
    d = _desc(T=0, n_rows=64, n_cols=64, K=4096, H=1 << 20)
    assert _product("omnimoe_grouped_product", d, _q(x_order=2), [(i, None) for i in range(5)]) == OK
    n = ctypes.c_size_t(1)
    size = _lib().omnimoe_grouped_product_dw_workspace_size
    assert size(ctypes.byref(d), ctypes.byref(_q(x_order=2)), ctypes.byref(n)) == OK and n.value == 0


# ------------------------------------------------------------------ the plain forms

@pytest.mark.parametrize("gate", [None, "token", "channel"])
@pytest.mark.parametrize("absent", ["", "w_out", "scale", "w_in", "y", "dx_out"])
def test_plain_join_gradients_match_differences(gate, absent):
    T, d, eps = 3, 5, 0.1
    g = torch.Generator().manual_seed(len(absent) + 7)
    names = ["x", "y", "gate", "w_out", "scale", "w_in"]
    shapes = dict(x=(T, d), y=(T, d), gate=(T, 1 if gate == "token" else d), w_out=(d,), scale=(d,), w_in=(d,))
    v = {k: torch.randn(shapes[k], generator=g, dtype=S.F64) for k in names}
    if gate is None:
        v["gate"] = None
    if absent in v:
        v[absent] = None
    da, dn = (torch.randn((T, d), generator=g, dtype=S.F64) for _ in range(2))
    if absent == "dx_out":
        da = None

    def loss(v):
        z, n = K.join(v["x"], v["y"], v["gate"], v["w_out"], v["scale"], v["w_in"], eps)
        return float((0 if da is None else (da * z).sum()) + (0 if n is None else (dn * n).sum()))

    z, _ = K.join(v["x"], v["y"], v["gate"], v["w_out"], v["scale"], v["w_in"], eps)
    got = K.join_back(z, v["y"], v["gate"], v["w_out"], v["scale"], v["w_in"], da, dn, eps)
    for k in names:
        if v[k] is None or (v["y"] is None and k in ("gate", "w_out", "scale")):
            continue
        grad = got["d" + k].reshape(-1)
        for i in range(v[k].numel()):
            h, w = 1e-5, {m: None if t is None else t.clone() for m, t in v.items()}
            w[k].view(-1)[i] += h
            up = loss(w)
            w[k].view(-1)[i] -= 2 * h
            diff = (up - loss(w)) / (2 * h)
            # a central difference's own error: h^2 / 6 of the third derivative and 2^-52 |loss| / h
            assert abs(diff - float(grad[i])) <= 2e-8 * (1 + abs(diff)), (k, i)


def test_plain_products_against_loops():
    g = torch.Generator().manual_seed(3)
    N, T, Kk, k, n = 5, 7, 2, 8, 6
    idx = torch.randint(0, 4, (T * Kk,), generator=g)  # expert 4 has none
    perm, offsets = K.schedule(idx, N)
    x, w, dy = (torch.randn(s, generator=g, dtype=S.F64) for s in ((T, k), (N, 2 * n, k), (T * Kk, 2 * n)))
    y, _ = K.product(x[K.rows_of(perm, "token", Kk, T * Kk, "cpu")], w, offsets, True, torch.float32)
    h, _ = K.product(x[K.rows_of(perm, "token", Kk, T * Kk, "cpu")], w, offsets, False, torch.float32)
    dw, _ = K.product_dw(x[K.rows_of(perm, "token", Kk, T * Kk, "cpu")], dy, offsets, torch.float32)
    dx, _ = K.product_dx(dy, w, offsets, torch.float32)
    sums = torch.zeros_like(w)
    for p, task in enumerate(perm.tolist()):
        e, t = int(idx[task]), task // Kk
        z = w[e] @ x[t]
        torch.testing.assert_close(h[p], z)
        torch.testing.assert_close(y[p], z[:n] * torch.sigmoid(z[:n]) * z[n:])
        torch.testing.assert_close(dx[p], dy[p] @ w[e])
        sums[e] += torch.outer(dy[p], x[t])
    torch.testing.assert_close(dw, sums)
    assert int(dw[4].count_nonzero()) == 0


def test_every_code_is_its_own_weight():
    codes = torch.arange(256, dtype=torch.uint8).repeat_interleave(16).view(1, 256, 16)
    codes[:, :, 1:] = 0x77  # 6 in every block, so that its scale is the power itself
    scales = torch.arange(2, 253, dtype=torch.uint8)[torch.arange(256) % 251].view(1, 256, 1)
    w = K.dequantise4(codes, scales)
    q, s = K.quantise4(w)
    assert torch.equal(q, w) and torch.equal(s, scales)


def test_nearest_codes_and_ties():
    row = [6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.2500001, 0.7499999, 4.9999, 5.0001, -0.25, -0.75, -5.0, 0.1]
    want = [6.0, 0.0, 1.0, 1.0, 2.0, 2.0, 4.0, 4.0, 0.5, 0.5, 4.0, 6.0, 0.0, -1.0, -4.0, 0.0]
    q, s = K.quantise4(torch.tensor([row + [0.0] * 16], dtype=S.F64))
    assert q[0, :16].tolist() == want and s.tolist() == [[127]]
