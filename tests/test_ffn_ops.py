"""The operators of include/omnimoe_ffn.h on the CPU: what the library exports, the refusals of every entry point (which
come from the host-side checks, before anything is launched), and the plain 64-bit forms that the GPU tests compare with."""
import ctypes
import os
import re

import pytest
import torch

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


def test_header_matches_exports():
    with open(os.path.join(ROOT, "include", "omnimoe_ffn.h")) as f:
        names = sorted(set(re.findall(r"^omnimoe_status\s+(omnimoe_\w+)\(", f.read(), flags=re.M)))
    assert sorted(P.EXPORTED_FFN) == names
    for n in names:
        assert hasattr(_lib(), n) and hasattr(P, n)


def test_adapter_descriptor_layout():
    # two int32, then five pointers
    assert ctypes.sizeof(B.OmnimoeAdapters) == 48 and B.OmnimoeAdapters.a_gu.offset == 8


def test_few_tokens_constant():
    with open(os.path.join(ROOT, "include", "omnimoe_ffn.h")) as f:
        assert int(re.search(r"#define OMNIMOE_FEW_TOKENS (\d+)", f.read()).group(1)) == P.FEW_TOKENS


def _desc(T=100, d=64, dtype=torch.bfloat16, **kw):
    return S.desc(T, d, dtype, **kw)


def _adapters(n=4, rank=8, ptr=0x10000, scale=0x10000):
    return B.OmnimoeAdapters(n=n, rank=rank, a_gu=ptr, b_gu=ptr, a_down=ptr, b_down=ptr, scale=scale)


def test_checkpoint_refusals():
    lib, D = _lib(), ctypes.byref(_desc())
    assert lib.omnimoe_checkpoint_store(D, None, A, A, None) == INVALID
    assert lib.omnimoe_checkpoint_store(D, A, A, None, None) == INVALID
    assert lib.omnimoe_checkpoint_store(D, A, BAD, A, None) == ALIGN
    assert lib.omnimoe_checkpoint_store(None, A, A, A, None) == INVALID
    assert lib.omnimoe_checkpoint_load(D, A, None, A, None) == INVALID
    assert lib.omnimoe_checkpoint_load(D, A, A, BAD, None) == ALIGN
    assert lib.omnimoe_checkpoint_load(ctypes.byref(_desc(d=60)), A, A, A, None) == INVALID
    none = ctypes.byref(_desc(T=0))
    assert lib.omnimoe_checkpoint_store(none, None, None, None, None) == OK
    assert lib.omnimoe_checkpoint_load(none, None, None, None, None) == OK


def _backward(desc, d_ff, change=(), ws=BIG):
    args = [A] * 10
    for i, v in change:
        args[i] = v
    return _lib().omnimoe_shared_mlp_backward(ctypes.byref(desc), d_ff, *args, ws, None)


def test_backward_refusals():
    # codes, scales, w_gu, w_down, dy, dx_in, dx, dw_gu, dw_down, workspace
    d = _desc()
    for i in (0, 1, 2, 3, 4, 6, 7, 8, 9):
        assert _backward(d, 64, [(i, None)]) == INVALID, i
    for i in range(10):
        assert _backward(d, 64, [(i, BAD)]) == ALIGN, i
    for d_ff in (0, 12, -8, 65544):
        assert _backward(d, d_ff) == INVALID
    assert _backward(d, 64, ws=ctypes.c_size_t(16)) == WORKSPACE
    assert _backward(_desc(T=-1), 64) == INVALID
    n = ctypes.c_size_t(0)
    size = _lib().omnimoe_shared_mlp_backward_workspace_size
    assert size(ctypes.byref(d), 64, None) == INVALID and size(ctypes.byref(d), 7, ctypes.byref(n)) == INVALID
    assert size(ctypes.byref(d), 64, ctypes.byref(n)) == OK
    # x, dy in two halves, dg and du, a: bf16
    assert n.value >= 100 * (3 * 64 + 3 * 64) * 2
    assert size(ctypes.byref(_desc(T=0)), 64, ctypes.byref(n)) == OK


def test_backward_workspace_holds_the_parts():
    # 4093 tokens, 512 wide: the weight gradients' sums are split; their parts lie in the workspace
    n = ctypes.c_size_t(0)
    assert _lib().omnimoe_shared_mlp_backward_workspace_size(ctypes.byref(_desc(T=4093, d=512)), 512,
                                                             ctypes.byref(n)) == OK
    assert n.value > 4093 * 6 * 512 * 2 + 512 * 512 * 4


def _adapt(desc, d_ff, ad, change=(), ws=BIG):
    args = [A] * 7  # x, w_gu, w_down, ids, y_in, y, workspace
    for i, v in change:
        args[i] = v
    return _lib().omnimoe_shared_mlp_adapters(ctypes.byref(desc), d_ff, None if ad is None else ctypes.byref(ad), *args,
                                              ws, None)


def test_adapter_refusals():
    d, ad = _desc(), _adapters()
    for i in (0, 1, 2, 3, 5, 6):
        assert _adapt(d, 64, ad, [(i, None)]) == INVALID, i
    for i in range(7):
        assert _adapt(d, 64, ad, [(i, BAD)]) == ALIGN, i
    assert _adapt(d, 64, None) == INVALID
    for n, rank, status in ((-1, 8, INVALID), (4, 0, INVALID), (4, 12, INVALID), (4, 264, INVALID),
                            (8193, 8, UNSUPPORTED)):
        assert _adapt(d, 64, _adapters(n, rank)) == status
    assert _adapt(d, 64, _adapters(ptr=None)) == INVALID
    assert _adapt(d, 64, _adapters(ptr=0x10004)) == ALIGN
    assert _adapt(d, 64, _adapters(scale=0x10004)) == ALIGN
    assert _adapt(d, 12, ad) == INVALID
    assert _adapt(d, 64, ad, ws=ctypes.c_size_t(16)) == WORKSPACE
    assert _adapt(_desc(T=10), 64, ad, ws=ctypes.c_size_t(16)) == WORKSPACE
    assert _adapt(_desc(T=0), 64, ad, [(i, None) for i in range(7)]) == OK
    n = ctypes.c_size_t(0)
    size = _lib().omnimoe_shared_mlp_adapters_workspace_size
    assert size(ctypes.byref(d), 64, ctypes.byref(ad), None) == INVALID
    assert size(ctypes.byref(d), 64, None, ctypes.byref(n)) == INVALID
    assert size(ctypes.byref(d), 64, ctypes.byref(_adapters(n=0, ptr=None, scale=None)), ctypes.byref(n)) == OK


def _few(desc, d_ff, change=(), ws=BIG):
    args = [A] * 11  # x, keys_row, keys_col, u, v, w_gu, w_down, y, idx, gates, workspace
    for i, v in change:
        args[i] = v
    return _lib().omnimoe_layer_forward_few(ctypes.byref(desc), d_ff, *args, ws, None)


def test_few_refusals():
    d = _desc(T=4, K=4)
    for i in (0, 1, 2, 3, 4, 5, 6, 7, 10):
        assert _few(d, 64, [(i, None)]) == INVALID, i
    for i in range(11):
        assert _few(d, 64, [(i, BAD)]) == ALIGN, i
    assert _few(_desc(T=17), 64) == UNSUPPORTED
    assert _few(_desc(T=4, K=65), 64) == UNSUPPORTED
    assert _few(d, 12) == INVALID and _few(d, -8) == INVALID
    assert _few(d, 64, ws=ctypes.c_size_t(16)) == WORKSPACE
    # without a shared branch its weights are not asked for
    assert _few(d, 0, [(5, None), (6, None)], ws=ctypes.c_size_t(16)) == WORKSPACE
    assert _few(_desc(T=0), 64, [(i, None) for i in range(11)]) == OK
    n = ctypes.c_size_t(0)
    size = _lib().omnimoe_layer_few_workspace_size
    assert size(ctypes.byref(_desc(T=17)), 64, ctypes.byref(n)) == UNSUPPORTED
    assert size(ctypes.byref(d), 64, None) == INVALID
    assert size(ctypes.byref(d), 0, ctypes.byref(n)) == OK


def test_binding_refuses_before_the_call():
    d = _desc(T=4)
    x, codes, scales = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8)
    with pytest.raises(ValueError, match="not on a GPU"):
        P.omnimoe_checkpoint_store(d, x, codes, scales)
    with pytest.raises(ValueError, match="float32"):
        P.omnimoe_checkpoint_store(d, x.float(), codes, scales)
    with pytest.raises(P.OmnimoeError):
        P.omnimoe_layer_few_workspace_size(_desc(T=17), 64)


def _bound_adapters_call(ad, T=4, d=64, f=72):
    x, w_gu, w_down = torch.zeros(T, d), torch.zeros(2 * f, d), torch.zeros(d, f)
    P.omnimoe_shared_mlp_adapters(_desc(T=T, d=d, dtype=torch.float32), f, ad, x, w_gu, w_down,
                                  torch.zeros(T, dtype=torch.int32), None, torch.zeros(T, d),
                                  ws=torch.zeros(256, dtype=torch.uint8))


def test_binding_of_a_descriptor_made_directly():
    # its tables are not known to the binding, so that it takes one without slots only
    with pytest.raises(ValueError, match="make_adapters"):
        _bound_adapters_call(_adapters())
    with pytest.raises(ValueError, match="not on a GPU"):  # the next refusal: these tensors are not
        _bound_adapters_call(B.OmnimoeAdapters(n=0, rank=8))


def test_binding_of_a_descriptor_changed_after_its_tables_were_checked():
    f, n, r, d = 72, 4, 8, 64
    tables = [torch.zeros(n, 2 * r, d), torch.zeros(n, 2 * f, r), torch.zeros(n, r, f), torch.zeros(n, d, r)]
    for name, value in (("n", n + 1), ("rank", 2 * r), ("rank", r // 2)):
        ad = P.make_adapters(*tables)
        setattr(ad, name, value)
        with pytest.raises(ValueError, match="tables made for 4 of rank 8"):
            _bound_adapters_call(ad)
    ad = P.make_adapters(*tables)
    ad.n = n - 1  # fewer slots: the first ones
    with pytest.raises(ValueError, match="not on a GPU"):
        _bound_adapters_call(ad)


def test_every_e4m3_value_is_its_own_checkpoint():
    # all finite codes, times powers of two from the least to the largest scale
    byte = torch.tensor([b for b in range(256) if b & 127 != 127], dtype=torch.uint8)
    v = S.dequantise(byte.view(1, -1), torch.full((1, 8), 127, dtype=torch.uint8))
    assert v.max() == 448 and torch.unique(v.abs()).numel() == 127
    rows = torch.cat([torch.cat((v[0], torch.tensor([448.0, -448.0], dtype=S.F64))) * 2.0 ** e for e in (-118, -3, 0, 100)]).view(4, 256)
    # every block of 32 holds its 448 so that its scale is the power itself
    rows = torch.cat((rows.view(4, -1, 16)[:, :, :15], torch.tensor([448.0 * 2.0 ** e for e in (-118, -3, 0, 100)], dtype=S.F64).view(4, 1, 1).expand(4, 16, 1)), 2)
    rows = torch.cat((rows, rows), 2).reshape(4, -1)
    q, s = S.quantise(rows)
    assert torch.equal(q, rows)
    assert s[:, 0].tolist() == [127 - 118, 127 - 3, 127, 227]


@pytest.mark.parametrize("seed", [0, 1])
def test_plain_backward_matches_differences(seed):
    T, d, f = 5, 6, 7
    g = torch.Generator().manual_seed(seed)
    x, wg, wd, dy = (torch.randn(s, generator=g, dtype=S.F64) for s in ((T, d), (2 * f, d), (d, f), (T, d)))

    def loss(x, wg, wd):
        h = x @ wg.t()
        return float((dy * ((S.silu(h[:, :f]) * h[:, f:]) @ wd.t())).sum())

    grads = S.mlp_backward(x, wg, wd, dy)
    for k, (v, grad) in enumerate(zip((x, wg, wd), grads)):
        for i in range(0, v.numel(), 5):
            args = [x.clone(), wg.clone(), wd.clone()]
            h = 1e-5
            args[k].view(-1)[i] += h
            up = loss(*args)
            args[k].view(-1)[i] -= 2 * h
            got = (up - loss(*args)) / (2 * h)
            # a central difference's own error: h^2 / 6 of the third derivative and 2^-52 |loss| / h
            assert abs(got - float(grad.reshape(-1)[i])) <= 1e-7 * (1 + abs(got))
