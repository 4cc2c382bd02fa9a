"""Where the gradients of the calls on rows of logits may lie: memory of their own, the logits', columns beside them."""
import numpy as np
import pytest

import paper_2510_15545_amd as tt
import util_rows as ur
from test_gpu_distill import compare
from test_rows_abi import PTR, backward, distill


@pytest.mark.parametrize("call", [backward, distill])
def test_rows_that_meet_are_refused(call):
    """Rows of 100 elements at a stride of 300, their gradients at the same stride or another one."""
    for size, dtype in ((2, 0), (4, 2)):
        for off in (1, 50, 99, 201, 250, 299, 301, 399, 300, 600, 899, -1, -99, -201, -299, -300, -399):
            assert call(n=4, ld=300, out=PTR + off * size, out_ld=300, dtype=dtype) == tt.TT_EINVAL, off
        for ld in (100, 200, 299, 301, 600):
            assert call(n=4, ld=300, out=PTR + 100 * size, out_ld=ld, dtype=dtype) == tt.TT_EINVAL, ld
        assert call(n=4, ld=100, out=PTR + 100 * size, out_ld=100, dtype=dtype) == tt.TT_EINVAL  # the next row


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("v", [37, 9001, 70001])
def test_gradients_beside_the_logits(v, dtype):
    """Logits and gradients as columns of one buffer, on either side, and as every other row of one."""
    import torch

    rng = np.random.default_rng(v)
    n, k = 5, 8
    x = torch.from_numpy(ur.model_rows(rng, n, v)).to(ur.torch_type(dtype)).cuda()
    ids = torch.from_numpy(rng.integers(0, v, n).astype(np.int32)).cuda()
    lists = ((ids[:, None] + 3 * torch.arange(k, device="cuda")) % v).int()
    lp, g = torch.randn((n, k), device="cuda") - 3, torch.randn(n, device="cuda")
    stats = tt.logprobs(v, x).stats
    want = tt.logprobs_backward(v, x, ids, stats, g)
    wide, tall = (lambda: torch.full((n, 2 * v + 3), 7.0, dtype=x.dtype, device="cuda")), (lambda: torch.full((2 * n, v), 7.0, dtype=x.dtype, device="cuda"))
    for make, at, to in ((wide, lambda b: b[:, :v], lambda b: b[:, v:2 * v]), (wide, lambda b: b[:, v + 3:], lambda b: b[:, 1:v + 1]),
                         (tall, lambda b: b[::2], lambda b: b[1::2]), (tall, lambda b: b[1::2], lambda b: b[::2])):
        for listed in (False, True):
            both = make()
            at(both).copy_(x)
            if listed:  # its sums' last digits go by the rows' alignment
                loss, grad = tt.distill(v, at(both), lists, lp, tail=True, grad_loss=g, dlogits=to(both))
                compare(loss, grad, ur.host(x), *(t.cpu().numpy() for t in (lists, lp)), None, True, g.cpu().numpy(), dtype)
            else:
                tt.logprobs_backward(v, at(both), ids, stats, g, out=to(both))
                assert torch.equal(to(both), want)
            rest = both.clone()
            at(rest).fill_(7.0)
            to(rest).fill_(7.0)
            assert (rest == 7.0).all()  # what lies beside the two is left alone
            assert torch.equal(at(both), x)
