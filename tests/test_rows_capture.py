"""A workspace that the calls on rows of logits make under capture: torch's graphs keep it, a capture begun outside
torch does not and has to be given one.  Split rows, captured and replayed."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2510_15545_amd as tt
import util_rows as ur
from test_rows_abi import PTR, fake


@pytest.mark.parametrize("capturing", [False, True])
@pytest.mark.parametrize("pool", [(0, 0), (0, 3)])
def test_a_capture_that_does_not_keep_the_workspace_is_refused(monkeypatch, capturing, pool):
    monkeypatch.setattr(torch, "empty", lambda *a, **k: fake(shape=(512,), dtype=torch.uint8))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: capturing)
    segments = [dict(address=PTR - 4096, total_size=4096, segment_pool_id=(0, 1)), dict(address=PTR - 512, total_size=2048, segment_pool_id=pool)]
    segments[0]["total_size"] = 4096 - 512
    monkeypatch.setattr(torch.cuda, "memory_snapshot", lambda: segments)
    if capturing and pool == (0, 0):
        with pytest.raises(ValueError, match="workspace"):
            tt._needed_workspace(None, 512, 0)
    else:
        assert tt._needed_workspace(None, 512, 0)[0] == PTR
    assert tt._needed_workspace(None, 0, 0) == (None, 0, None)


N, V, K = 5, 70001, 24  # rows that are split


def inputs(seed):
    rng = np.random.default_rng(seed)
    rows = ur.placed(ur.model_rows(rng, N, V), "bf16")
    ids = torch.from_numpy(np.stack([rng.choice(V, K, replace=False) for _ in range(N)]).astype(np.int32)).cuda()
    return rows, ids, torch.randn((N, K), device="cuda") - 4, torch.rand(N, device="cuda")


def calls(rows, ids, lp, w, f=None, loss=None, grad=None, **kw):
    one = ids[:, 0].contiguous()
    spaces = kw.get("spaces", (None, None))
    f = tt.logprobs(V, rows, one, n_top=K, entropy=True, out=f, workspace=spaces[0])
    return [*f, *tt.distill(V, rows, ids, lp, tail=True, grad_loss=w, loss=loss, dlogits=grad, workspace=spaces[1])]


@pytest.mark.gpu
@pytest.mark.parametrize("given", ["nothing", "outputs", "all"])
def test_split_rows_replayed_in_a_graph_on_new_inputs(given):
    held = inputs(1)
    kw = {}
    if given != "nothing":
        first = calls(*held)
        kw = dict(f=tt.LogProbs(*(torch.empty_like(t) for t in first[:6])), loss=torch.empty_like(first[6]), grad=torch.empty_like(first[7]))
    if given == "all":
        kw["spaces"] = tt.logprobs_workspace(N, V, torch.bfloat16, K), tt.distill_workspace(N, V, torch.bfloat16, K, grad=True)
        assert all(s.numel() > 0 for s in kw["spaces"])
    calls(*held, **kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        results = calls(*held, **kw)
    for seed in range(2, 6):
        for old, new in zip(held, inputs(seed)):
            old.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, calls(*held))), seed


@pytest.mark.gpu
def test_a_capture_begun_outside_torch():
    """Nothing of it is replayed: the calls without a workspace raise, those with one are recorded."""
    held = inputs(1)
    want = calls(*held)
    f, loss, grad = tt.LogProbs(*(torch.empty_like(t) for t in want[:6])), torch.empty_like(want[6]), torch.empty_like(want[7])
    spaces = tt.logprobs_workspace(N, V, torch.bfloat16, K), tt.distill_workspace(N, V, torch.bfloat16, K, grad=True)
    one = held[1][:, 0].contiguous()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):  # memory of the stream's pool that the refused calls can take and give back
        torch.empty(spaces[0].numel(), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    hip, stream = tt.lib(), ctypes.c_void_p(side.cuda_stream)
    graph, nodes = ctypes.c_void_p(), ctypes.c_size_t(0)
    relaxed = 2
    with torch.cuda.stream(side):
        assert hip.hipStreamBeginCapture(stream, relaxed) == 0
        try:
            with pytest.raises(ValueError, match="workspace"):
                tt.logprobs(V, held[0], one, n_top=K, out=f)
            with pytest.raises(ValueError, match="workspace"):
                tt.distill(V, *held[:3], tail=True, grad_loss=held[3], loss=loss, dlogits=grad)
            tt.logprobs(V, held[0], one, n_top=K, out=f, workspace=spaces[0])
            tt.distill(V, *held[:3], tail=True, grad_loss=held[3], loss=loss, dlogits=grad, workspace=spaces[1])
        finally:
            assert hip.hipStreamEndCapture(stream, ctypes.byref(graph)) == 0
    assert hip.hipGraphGetNodes(graph, None, ctypes.byref(nodes)) == 0
    assert nodes.value == 5  # two kernels and three
    assert hip.hipGraphDestroy(graph) == 0
    assert all(torch.equal(a, b) for a, b in zip(want, calls(*held)))
