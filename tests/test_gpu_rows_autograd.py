"""Memory of the caller's that the calls on rows of logits write, as torch's autograd sees it: what was saved for a
backward pass and overwritten since is an error, what was not saved may be overwritten."""
import pytest
import torch

import paper_2510_15545_amd as tt

pytestmark = pytest.mark.gpu

N, V, K = 6, 4001, 8
SPOILT = "modified by an inplace operation"


def inputs():
    gen = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((N, V), device="cuda", generator=gen)
    ids = torch.randint(0, V, (N, K), device="cuda", generator=gen, dtype=torch.int32)
    lp = torch.randn((N, K), device="cuda", generator=gen) - 3
    return x, ids, lp, torch.rand(N, device="cuda", generator=gen)


def gradients(ids, lp, g):
    """(name, call): the gradient of rows, in memory of its own or in `to`."""
    return (("backward", lambda rows, to: tt.logprobs_backward(V, rows, ids[:, 0].contiguous(), tt.logprobs(V, rows).stats, g, out=to)),
            ("distill", lambda rows, to: tt.distill(V, rows, ids, lp, tail=True, grad_loss=g, dlogits=to)[1]))


def test_gradients_over_logits_that_an_operation_saved():
    """A soft cap's result is what its backward pass takes."""
    x, *more = inputs()
    for name, call in gradients(*more):
        leaf = x.clone().requires_grad_()
        logits = torch.tanh(leaf)
        grad = call(logits.detach(), logits.detach())
        with pytest.raises(RuntimeError, match=SPOILT):
            logits.backward(grad)
        logits = torch.tanh(leaf)
        logits.backward(call(logits.detach(), None))
        assert leaf.grad.any(), name


def test_gradients_over_logits_that_no_operation_saved():
    x, *more = inputs()
    hidden = torch.randn((N, 32), device="cuda")
    for name, call in gradients(*more):
        got = []
        for in_place in (False, True):
            head = torch.ones((V, 32), device="cuda").mul_(x[0, :, None]).requires_grad_()
            logits = hidden @ head.t()
            logits.backward(call(logits.detach(), logits.detach() if in_place else None))
            got.append(head.grad)
        assert torch.equal(*got), name


def test_results_in_the_callers_memory():
    x, ids, lp, g = inputs()
    out = tt.logprobs(V, x, ids[:, 0].contiguous(), n_top=K, entropy=True)
    for name in ("logprob", "lse", "stats", "entropy", "top_logprobs"):
        scale = torch.ones(1, device="cuda", requires_grad=True)
        y = (getattr(out, name) * scale).sum()
        tt.logprobs(V, x, ids[:, 0].contiguous(), n_top=K, out=out)
        with pytest.raises(RuntimeError, match=SPOILT):
            y.backward()
    loss, _ = tt.distill(V, x, ids, lp)
    scale = torch.ones(1, device="cuda", requires_grad=True)
    y = (loss * scale).sum()
    tt.distill(V, x, ids, lp, loss=loss)
    with pytest.raises(RuntimeError, match=SPOILT):
        y.backward()


def test_inference_tensors_have_no_versions():
    x, *more = inputs()
    with torch.inference_mode():
        for name, call in gradients(*more):
            rows = x.clone()
            want = call(rows, None)
            assert torch.equal(call(rows, rows), want), name
