"""Refusals of the calls on rows of logits, before anything is launched: sizes, types, strides, alignment, pointers,
workspaces, overlapping gradients, and the binding's checks of its tensors."""
import ctypes
import types

import pytest
import torch

import paper_2510_15545_amd as tt

L = tt.lib()
PTR = 0x100000000  # never read: every call below is refused


def logprobs(n=2, v=100, dtype=0, logits=PTR, ld=100, temp=None, ids=PTR, n_top=3, logprob=PTR, lse=PTR, stats=PTR, entropy=PTR,
             top_ids=PTR, top_lp=PTR, ws=PTR, nbytes=1 << 30):
    return L.tt_logprobs(n, v, dtype, logits, ld, temp, ids, n_top, logprob, lse, stats, entropy, top_ids, top_lp, ws, nbytes, None)


def backward(n=2, v=100, dtype=0, logits=PTR, ld=100, temp=None, ids=PTR, stats=PTR, entropy=None, g=PTR, h=None, out=2 * PTR, out_ld=100):
    return L.tt_logprobs_backward(n, v, dtype, logits, ld, temp, ids, stats, entropy, g, h, out, out_ld, None)


def distill(n=2, v=100, dtype=0, logits=PTR, ld=100, temp=None, k=3, ids=PTR, lp=PTR, id_map=None, n_map=0, tail=0, loss=PTR, g=PTR,
            out=2 * PTR, out_ld=100, ws=PTR, nbytes=1 << 30):
    return L.tt_distill(n, v, dtype, logits, ld, temp, k, ids, lp, id_map, n_map, tail, loss, g, out, out_ld, ws, nbytes, None)


@pytest.mark.parametrize("call", [logprobs, backward, distill])
def test_sizes_types_and_pointers(call):
    for bad in (dict(n=-1), dict(v=0), dict(v=-5), dict(dtype=3), dict(dtype=-1), dict(ld=99), dict(logits=None),
                dict(logits=PTR + 1), dict(dtype=2, logits=PTR + 2), dict(ld=1 << 62), dict(n=2 ** 31 - 1, ld=1 << 33)):
        assert call(**bad) == tt.TT_EINVAL, bad
    assert call(v=(1 << 23) + 1, ld=1 << 24) in (tt.TT_EUNSUPPORTED, tt.TT_EINVAL)
    assert call(n=0, logits=None) == tt.TT_OK


def test_logprobs_refusals():
    for bad in (dict(n_top=-1), dict(ids=None), dict(top_ids=None), dict(top_lp=None)):
        assert logprobs(**bad) == tt.TT_EINVAL, bad
    assert logprobs(n_top=129) == tt.TT_EUNSUPPORTED
    assert logprobs(v=(1 << 23) + 1, ld=1 << 24) == tt.TT_EUNSUPPORTED
    n = ctypes.c_size_t(0)
    assert L.tt_logprobs_workspace_size(2, 100, 0, 3, ctypes.byref(n)) == tt.TT_OK and n.value == 0  # a row whole in a workgroup
    assert L.tt_logprobs_workspace_size(2, 100000, 0, 3, ctypes.byref(n)) == tt.TT_OK and n.value > 0
    assert logprobs(v=100000, ld=100000, nbytes=n.value - 1) == tt.TT_EWORKSPACE
    assert logprobs(v=100000, ld=100000, ws=None) == tt.TT_EWORKSPACE
    assert logprobs(v=100000, ld=100000, ws=PTR + 8) == tt.TT_EINVAL
    for bad in ((-1, 100, 0, 3), (2, 0, 0, 3), (2, 100, 5, 3), (2, 100, 0, -1)):
        assert L.tt_logprobs_workspace_size(*bad, ctypes.byref(n)) == tt.TT_EINVAL
    assert L.tt_logprobs_workspace_size(2, 100, 0, 129, ctypes.byref(n)) == tt.TT_EUNSUPPORTED
    assert L.tt_logprobs_workspace_size(2, (1 << 23) + 1, 0, 1, ctypes.byref(n)) == tt.TT_EUNSUPPORTED
    assert L.tt_logprobs_workspace_size(2, 100, 0, 3, None) == tt.TT_EINVAL
    assert L.tt_logprobs_workspace_size(0, 100, 0, 3, ctypes.byref(n)) == tt.TT_OK
    # the largest sizes: the rows' groups bound the workspace
    assert L.tt_logprobs_workspace_size(2 ** 31 - 1, 1 << 23, 2, 128, ctypes.byref(n)) == tt.TT_OK and n.value < 1 << 28


def test_backward_refusals():
    for bad in (dict(stats=None), dict(out=None), dict(out_ld=99), dict(ids=None), dict(g=None), dict(entropy=PTR), dict(h=PTR),
                dict(out=2 * PTR + 1), dict(out_ld=1 << 62)):
        assert backward(**bad) == tt.TT_EINVAL, bad
    # memory that overlaps the logits, but for the logits themselves
    for bad in (dict(out=PTR + 2), dict(out=PTR, out_ld=101), dict(out=PTR + 398), dict(out=PTR - 398), dict(out=PTR - 2)):
        assert backward(**bad) == tt.TT_EINVAL, bad


def test_distill_refusals():
    for bad in (dict(k=0), dict(k=-1), dict(ids=None), dict(lp=None), dict(loss=None), dict(g=None), dict(n_map=-1), dict(out_ld=99),
                dict(out=2 * PTR + 1), dict(out=PTR + 2), dict(out=PTR, out_ld=101)):
        assert distill(**bad) == tt.TT_EINVAL, bad
    assert distill(k=129) == tt.TT_EUNSUPPORTED
    assert distill(v=(1 << 23) + 1, ld=1 << 24, out_ld=1 << 24) == tt.TT_EUNSUPPORTED
    n = ctypes.c_size_t(0)
    assert L.tt_distill_workspace_size(2, 100, 0, 3, 1, ctypes.byref(n)) == tt.TT_OK and n.value == 0  # a row whole in a workgroup
    for grad, out in ((1, 2 * PTR), (0, None)):
        assert L.tt_distill_workspace_size(2, 100000, 0, 3, grad, ctypes.byref(n)) == tt.TT_OK and n.value > 0
        split = dict(v=100000, ld=100000, out=out, out_ld=100000)
        assert distill(nbytes=n.value - 1, **split) == tt.TT_EWORKSPACE
        assert distill(ws=None, **split) == tt.TT_EWORKSPACE
        assert distill(ws=PTR + 8, **split) == tt.TT_EINVAL
    for bad in ((-1, 100, 0, 3, 0), (2, 0, 0, 3, 0), (2, 100, 5, 3, 0), (2, 100, 0, 0, 0)):
        assert L.tt_distill_workspace_size(*bad, ctypes.byref(n)) == tt.TT_EINVAL
    assert L.tt_distill_workspace_size(2, 100, 0, 3, 0, None) == tt.TT_EINVAL
    assert L.tt_distill_workspace_size(2 ** 31 - 1, 1 << 23, 2, 128, 1, ctypes.byref(n)) == tt.TT_OK and n.value < 1 << 28


def test_host_tensors_and_wrong_shapes_are_refused():
    x, ids, f = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32), torch.zeros(2)
    with pytest.raises(ValueError):
        tt.logprobs(8, x, ids)
    with pytest.raises(ValueError):
        tt.logprobs_backward(8, x, ids, f, f)
    with pytest.raises(ValueError):
        tt.distill(8, x, ids.view(2, 1), f.view(2, 1))
    with pytest.raises(ValueError):
        tt.logprobs_workspace(2, 8, torch.float64)
    with pytest.raises(ValueError):
        tt.distill_workspace(2, 8, "int8", 4)


def fake(shape=(2, 8), dtype=torch.bfloat16, device=0, strides=None, contiguous=True):
    strides = strides or (shape[-1], 1)
    n = 1
    for s in shape:
        n *= s
    return types.SimpleNamespace(dim=lambda: len(shape), stride=lambda i: strides[i], is_cuda=True, dtype=dtype, shape=shape,
                                 numel=lambda: n, is_contiguous=lambda: contiguous, data_ptr=lambda: PTR, element_size=lambda: 2,
                                 get_device=lambda: device)


def test_devices_and_shapes_of_device_tensors(monkeypatch):
    """Tensors of another device than the current one or the stream's, of another size, type or layout: refused by the binding."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    assert tt._launch_device(fake(), None) == 0
    with pytest.raises(ValueError, match="current device"):
        tt._launch_device(fake(device=1), None)
    with pytest.raises(ValueError, match="stream belongs"):
        tt._launch_device(fake(), types.SimpleNamespace(cuda_stream=1, device_index=1))
    assert tt._launch_device(fake(device=1), types.SimpleNamespace(cuda_stream=1, device_index=1)) == 1
    assert tt._launch_device(fake(), types.SimpleNamespace(cuda_stream=1)) == 0
    assert tt._rows(fake(), 8, 2, "logits") == (0, PTR, 8)
    assert tt._rows(fake(shape=(1, 9), strides=(1, 1), dtype=torch.float32), 8, 1, "logits") == (2, PTR, 8)
    for bad, why in ((dict(dtype=torch.float64), "bfloat16, float16 or float32"), (dict(strides=(1, 2)), "row-major"),
                     (dict(shape=(2, 7)), "at least"), (dict(shape=(1, 8)), "at least"), (dict(shape=(16,), strides=(1, 1)), "row-major")):
        with pytest.raises(ValueError, match=why):
            tt._rows(fake(**bad), 8, 2, "logits")
    ids = dict(shape=(2,), dtype=torch.int32)
    assert tt._array(fake(**ids), torch.int32, 2, "ids", 0) == PTR and tt._array(None, torch.int32, 2, "ids", 0) is None
    for bad, why in ((dict(ids, shape=(3,)), "elements"), (dict(ids, dtype=torch.int64), "int32"), (dict(ids, contiguous=False), "contiguous"),
                     (dict(ids, device=1), "cuda:1")):
        with pytest.raises(ValueError, match=why):
            tt._array(fake(**bad), torch.int32, 2, "ids", 0)
    with pytest.raises(ValueError, match="workspace"):
        tt._needed_workspace(fake(device=1), 16, 0)
    with pytest.raises(ValueError, match="required"):
        tt.logprobs_backward(8, fake(), fake(**ids), None, fake(shape=(2,), dtype=torch.float32), out=fake())
