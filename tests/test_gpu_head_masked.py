"""Gradients of the output head where tokens are masked by weights of minus infinity."""
import pytest
import torch

import paper_2510_15545_amd as tt
import util_head as uh
from test_gpu_head import close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n", [1, 3, 32, 33, 64, 70, 100, 128, 130, 300])
def test_masked_tokens_have_no_gradient(n, name):
    """Their rows of dweight are zeros, whatever the rows' number; the others' are those of the vocabulary without them."""
    v, h = 1000, 40
    x, w, ids, beta = uh.operands(n, v, h, name)
    x[:, 1] = x[:, 1].abs() + 0.25
    w[:, 1] = 0.0
    masked = torch.zeros(v, dtype=torch.bool, device="cuda")
    masked[[0, 130, 400, 401, 870, 999]] = True
    keep = torch.nonzero(~masked)[:, 0]
    ids = keep[ids.long() % len(keep)].int()  # none of them a masked one
    w2 = w.clone()
    w2[masked, 1] = -float("inf")
    gen = torch.Generator().manual_seed(n)
    g = (torch.rand(n, generator=gen) + 0.5).cuda()
    q = torch.randn(n, generator=gen).cuda()
    place = torch.cumsum(~masked, 0) - 1
    for out in (0, n // 3):  # some rows without a weight
        some = ids.clone()
        some[:out] = -1
        weights = q.clone()
        weights[:out] = 0.0
        stats = tt.head_logprobs(v, x, w2, some, inv_temperature=beta).stats
        assert bool(torch.isfinite(stats).all())
        _, dw = tt.head_logprobs_backward(v, x, w2, some, stats, g, grad_lse=weights, inv_temperature=beta, dhidden=False)
        assert not bool(dw[masked].any())
        small = torch.where(some >= 0, place[some.long().clamp_min(0)], some.long()).int()
        _, want, _, off = uh.backward(x, w[keep], small, stats, g, weights, beta, name)
        close(dw[keep], want, off, f"dweight, {out} rows without a weight")
