"""The output head's gradient in fp16, whose range is short."""
import pytest
import torch

import paper_2510_15545_amd as tt
import util_head as uh

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("out", [0, 17])
@pytest.mark.parametrize("n", [50, 100])
def test_fp16_row_weights_of_very_different_sizes(n, out):
    """fp16 holds a row's gradient of the logits to 2^-39 of the largest row weight: rows of any weight and flat ones, whose
    probabilities are all small, with weights of the log-sum-exp beside them."""
    v, h = 2000, 64
    x, w, ids, beta = uh.operands(n, v, h, "f16")
    x[::5] = 0.0  # flat: 1 / v
    g = torch.logspace(-9, 3, n).cuda()
    q = -2.0 * torch.logspace(3, -9, n).cuda()
    ids[:out] = -1
    stats = tt.head_logprobs(v, x, w, ids, inv_temperature=beta).stats
    for weights in (None, q):
        got = tt.head_logprobs_backward(v, x, w, ids, stats, g, grad_lse=weights, inv_temperature=beta)
        want = uh.backward(x, w, ids, stats, g, weights, beta, "f16")
        for a, b, off in zip(got, want[:2], want[2:]):
            assert bool(((a.double() - b).abs() <= off).all())
