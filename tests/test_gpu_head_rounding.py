"""Errors of the output head's results as a whole: 16-bit gradients are those of one rounding of the result, whatever the rows'
number; equal calls give equal results."""
import pytest
import torch

import paper_2510_15545_amd as tt
import util_head as uh

pytestmark = pytest.mark.gpu


def gradients(n, v, h, name, out=0.0):
    """(the kernels' gradients, those in 64 bits) with the given share of rows without a weight."""
    x, w, ids, beta = uh.operands(n, v, h, name)
    gen = torch.Generator().manual_seed(n)
    g = (torch.rand(n, generator=gen) + 0.5).cuda()
    ids[torch.randperm(n, generator=gen)[:int(out * n)].cuda()] = -1
    stats = tt.head_logprobs(v, x, w, ids, inv_temperature=beta).stats
    call = lambda: tt.head_logprobs_backward(v, x, w, ids, stats, g, inv_temperature=beta)  # noqa: E731
    return call(), uh.backward(x, w, ids, stats, g, None, beta, name)[:2], call


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("n,v,h,out", [(1, 3000, 64, 0.0), (40, 3000, 64, 0.0), (65, 1000, 64, 0.0), (66, 3000, 96, 0.0), (100, 5000, 64, 0.3), (130, 2000, 65, 0.0),
                                       (300, 3000, 64, 0.5), (391, 4001, 64, 0.3), (520, 3000, 64, 0.0), (600, 6000, 128, 0.0)])
def test_gradients_are_rounded_once(n, v, h, out, name):
    """A result RN(y) of y = want + d is off by at most |RN(want) - want| + 2 |d|, value by value (RN(y) is the nearest to y, so no
    further from it than RN(want)).  d is what twice the type's digits of the logits' gradient leave (HALF_STEP^2 of every
    term) and what fp32 sums of 64 to 128 products and their exponentials do, about 16 U of logits of up to 16: under a
    thirty-second of HALF_STEP even in fp16 (2^-16 against 2^-11)."""
    got, want, again = gradients(n, v, h, name, out)
    for a, b, what in zip(got, want, ("dhidden", "dweight")):
        once = float((b.to(a.dtype).double() - b).norm() / b.norm())
        off = float((a.double() - b).norm() / b.norm())
        assert off <= once + uh.HALF_STEP[name] / 16, (what, off, once)
    assert all(torch.equal(a, b) for a, b in zip(got, again()))
