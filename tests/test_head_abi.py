"""Refusals of the calls on the output head and of the 8-bit product, before anything is launched, and their workspaces."""
import ctypes

import pytest
import torch

import paper_2510_15545_amd as tt
from test_rows_abi import fake

L = tt.lib()
PTR = 0x100000000  # never read: every call below is refused
BIG = 1 << 40


def forward(n=2, v=100, h=8, dtype=0, x=PTR, x_ld=8, w=2 * PTR, w_ld=8, temp=None, ids=PTR, logprob=PTR, lse=PTR, stats=PTR, ws=PTR, nbytes=BIG):
    return L.tt_head_logprobs(n, v, h, dtype, x, x_ld, w, w_ld, temp, ids, logprob, lse, stats, ws, nbytes, None)


def backward(n=2, v=100, h=8, dtype=0, x=PTR, x_ld=8, w=2 * PTR, w_ld=8, temp=None, ids=PTR, stats=PTR, g=PTR, q=None, dx=3 * PTR, dx_ld=8,
             dw=4 * PTR, dw_ld=8, ws=PTR, nbytes=BIG):
    return L.tt_head_logprobs_backward(n, v, h, dtype, x, x_ld, w, w_ld, temp, ids, stats, g, q, dx, dx_ld, dw, dw_ld, ws, nbytes, None)


def quantize(n=2, k=8, dtype=0, x=PTR, x_ld=8, q=2 * PTR, q_ld=8, scale=PTR):
    return L.tt_quantize_i8(n, k, dtype, x, x_ld, q, q_ld, scale, None)


def matmul(n=2, m=100, k=8, x=PTR, x_ld=8, xs=PTR, w=2 * PTR, w_ld=8, ws=PTR, bias=None, dtype=0, out=3 * PTR, out_ld=100, temp=None, lse=PTR,
           space=PTR, nbytes=BIG):
    return L.tt_matmul_i8(n, m, k, x, x_ld, xs, w, w_ld, ws, bias, dtype, out, out_ld, temp, lse, space, nbytes, None)


@pytest.mark.parametrize("call", [forward, backward])
def test_sizes_types_and_pointers(call):
    for bad in (dict(n=-1), dict(v=0), dict(h=0), dict(h=-3), dict(dtype=3), dict(dtype=-1), dict(x_ld=7), dict(w_ld=7), dict(x=None),
                dict(w=None), dict(x=PTR + 1), dict(w=2 * PTR + 1), dict(dtype=2, x=PTR + 2), dict(x_ld=1 << 62), dict(w_ld=1 << 62),
                dict(x_ld=1 << 56), dict(w_ld=1 << 56), dict(ws=PTR + 8), dict(ids=PTR + 2), dict(stats=PTR + 2)):
        assert call(**bad) == tt.TT_EINVAL, bad
    for big in (dict(n=(1 << 20) + 1), dict(v=(1 << 23) + 1), dict(h=(1 << 16) + 1, x_ld=1 << 17, w_ld=1 << 17, **({"dx_ld": 1 << 17, "dw_ld": 1 << 17} if call is backward else {}))):
        assert call(**big) == tt.TT_EUNSUPPORTED, big
    for small in (dict(ws=None), dict(nbytes=0), dict(nbytes=100)):
        assert call(**small) == tt.TT_EWORKSPACE, small


def test_forward_refusals():
    assert forward(n=0, x=None, w=None, ws=None) == tt.TT_OK
    assert forward(ids=None) == tt.TT_EINVAL


def test_backward_refusals():
    for bad in (dict(stats=None), dict(ids=None), dict(g=None), dict(dx=None, dw=None), dict(dx_ld=7), dict(dw_ld=7), dict(dx=3 * PTR + 1),
                dict(dw=4 * PTR + 1), dict(dx_ld=1 << 62), dict(dw_ld=1 << 62), dict(q=PTR + 1)):
        assert backward(**bad) == tt.TT_EINVAL, bad
    # gradients that meet an operand or each other, from either side; columns beside them in one buffer do not
    for bad in (dict(dx=PTR), dict(dx=PTR + 16), dict(dx=PTR - 16), dict(dw=2 * PTR), dict(dw=2 * PTR - 2), dict(dx=2 * PTR + 100),
                dict(dw=PTR - 1500), dict(dw=3 * PTR - 2), dict(x_ld=20, dx=PTR + 14, dx_ld=20), dict(x_ld=20, dx=PTR + 26, dx_ld=20)):
        assert backward(**bad) == tt.TT_EINVAL, bad
    for fine in (dict(x_ld=20, dx=PTR + 16, dx_ld=20), dict(x_ld=20, dx=PTR - 16, dx_ld=20), dict(w_ld=16, dw=2 * PTR + 16, dw_ld=16)):
        assert backward(nbytes=0, **fine) == tt.TT_EWORKSPACE, fine
    assert backward(n=0, x=None, dw=None) == tt.TT_OK
    assert backward(n=0, x=None, dw=4 * PTR + 1) == tt.TT_EINVAL


def test_quantize_refusals():
    for bad in (dict(n=-1), dict(k=0), dict(dtype=3), dict(x_ld=7), dict(q_ld=7), dict(x=None), dict(q=None), dict(scale=None), dict(x=PTR + 1),
                dict(scale=PTR + 2), dict(x_ld=1 << 62), dict(q_ld=1 << 62), dict(q=PTR), dict(q=PTR + 15), dict(q=PTR - 15)):
        assert quantize(**bad) == tt.TT_EINVAL, bad
    assert quantize(k=1 << 17, x_ld=1 << 17, q_ld=1 << 17) == tt.TT_EUNSUPPORTED
    assert quantize(n=0, x=None) == tt.TT_OK


def test_matmul_refusals():
    for bad in (dict(n=-1), dict(m=0), dict(k=0), dict(dtype=3), dict(x_ld=7), dict(w_ld=7), dict(out_ld=99), dict(x=None), dict(w=None),
                dict(xs=None), dict(ws=None), dict(out=None), dict(out=3 * PTR + 1), dict(xs=PTR + 1), dict(lse=PTR + 2), dict(space=PTR + 4),
                dict(out=PTR), dict(out=2 * PTR + 700), dict(out=2 * PTR - 300), dict(out_ld=1 << 62), dict(x_ld=1 << 62), dict(bias=PTR + 1)):
        assert matmul(**bad) == tt.TT_EINVAL, bad
    for big in (dict(k=1 << 17, x_ld=1 << 17, w_ld=1 << 17), dict(n=(1 << 20) + 1), dict(m=(1 << 23) + 1, out_ld=1 << 24)):
        assert matmul(**big) == tt.TT_EUNSUPPORTED, big
    for small in (dict(space=None), dict(nbytes=15)):
        assert matmul(**small) == tt.TT_EWORKSPACE, small
    assert matmul(n=0, x=None) == tt.TT_OK


def query(name, *sizes):
    n = ctypes.c_size_t(0)
    assert getattr(L, name)(*sizes, ctypes.byref(n)) == tt.TT_OK
    return n.value


ROWS = [1, 2, 7, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 200, 255, 256, 257, 300, 511, 513, 700, 1024, 1025, 2048, 3000, 4096, 9000, 70000]


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("v,h", [(640, 256), (50257, 1024), (151936, 2048), (300007, 64), (1, 1), (1000, 8192)])
def test_a_workspace_for_more_rows_serves_fewer(v, h, dtype):
    for op, used in (("tt_head_logprobs", "workspace_size"), ("tt_head_logprobs_backward", "workspace_used")):
        size = [query(f"{op}_workspace_size", n, v, h, dtype) for n in ROWS]
        assert size == sorted(size)
        most = 0
        for n, s in zip(ROWS, size):
            most = max(most, query(f"{op}_{used}", n, v, h, dtype))
            assert most <= s, (op, n)
    for lse in (0, 1):
        size = [query("tt_matmul_i8_workspace_size", n, v, h, lse) for n in ROWS]
        assert size == sorted(size)


def test_workspace_refusals():
    n = ctypes.c_size_t(0)
    for f in (L.tt_head_logprobs_workspace_size, L.tt_head_logprobs_backward_workspace_size, L.tt_head_logprobs_backward_workspace_used):
        for bad in ((-1, 100, 8, 0), (2, 0, 8, 0), (2, 100, 0, 0), (2, 100, 8, 3)):
            assert f(*bad, ctypes.byref(n)) == tt.TT_EINVAL
        assert f(2, (1 << 23) + 1, 8, 0, ctypes.byref(n)) == tt.TT_EUNSUPPORTED
        assert f(2, 100, 8, 0, None) == tt.TT_EINVAL
        assert f(0, 100, 8, 0, ctypes.byref(n)) == tt.TT_OK and n.value == 0
        assert f(1 << 20, 1 << 23, 1 << 16, 2, ctypes.byref(n)) == tt.TT_OK and n.value > 0
    assert L.tt_matmul_i8_workspace_size(2, 100, 1 << 17, 0, ctypes.byref(n)) == tt.TT_EUNSUPPORTED
    assert L.tt_matmul_i8_workspace_size(2, 100, 8, 0, None) == tt.TT_EINVAL


def test_bindings_checks(monkeypatch):
    x, w, f = torch.zeros(2, 8), torch.zeros(9, 8), torch.zeros(2)
    with pytest.raises(ValueError):
        tt.head_logprobs(9, x, w)
    with pytest.raises(ValueError):
        tt.quantize_i8(x)
    with pytest.raises(ValueError):
        tt.matmul_i8(x.to(torch.int8), f, w.to(torch.int8), torch.zeros(9))
    with pytest.raises(ValueError):
        tt.head_logprobs_workspace(2, 9, 8, torch.float64)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    assert tt._head(9, fake(), fake(shape=(9, 8)), None)[:3] == (2, 8, 0)
    for bad, why in ((fake(shape=(9, 7)), "at least"), (fake(shape=(9, 9)), "rows of 8"), (fake(shape=(8, 8)), "at least"),
                     (fake(shape=(9, 8), dtype=torch.float16), "rows of 8"), (fake(shape=(9, 8), device=1), "cuda:1"), (fake(shape=(9,)), "2-D")):
        with pytest.raises(ValueError, match=why):
            tt._head(9, fake(), bad, None)
    i8 = dict(dtype=torch.int8)
    assert tt._bytes(fake(**i8), "x", 0)[1] == 8
    for bad, why in ((fake(), "int8"), (fake(shape=(8,), strides=(1, 1), **i8), "2-D"), (fake(strides=(1, 2), **i8), "row-major"), (fake(device=1, **i8), "cuda:1")):
        with pytest.raises(ValueError, match=why):
            tt._bytes(bad, "x", 0)
