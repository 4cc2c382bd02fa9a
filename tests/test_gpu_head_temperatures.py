"""Gradients of the output head at inverse temperatures where a rounding of a logit is many units of the exponent."""
import pytest
import torch

import paper_2510_15545_amd as tt
import util_head as uh

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 5, 16, 40, 64, 70, 300])
@pytest.mark.parametrize("power", [20, 60, 100])
def test_probabilities_stay_below_one(n, power, name):
    """Wherever the rounding of the largest logit falls, its p lies in [0, 1], and that of the others is 0."""
    v, h, beta = 700, 512, 2.0 ** power
    x, w, ids, _ = uh.operands(n, v, h, name, seed=3)
    top = (x.double() @ w.double().T).argmax(1)  # the next logit is units away
    b = torch.full((n,), beta, device="cuda")
    g = torch.ones(n, device="cuda")
    stats = tt.head_logprobs(v, x, w, ids, inv_temperature=b).stats
    dx, dw = tt.head_logprobs_backward(v, x, w, ids, stats, g, inv_temperature=b)
    assert bool(torch.isfinite(dx.float()).all()) and bool(torch.isfinite(dw.float()).all())
    # dz is beta at the token and minus beta p at the largest logit, p in [0, 1]; half a step each for dz, twice, and the result
    wd = w.double().abs()
    room = (1 + 4 * uh.HALF_STEP[name]) * beta
    assert bool((dx.double().abs() <= room * (wd[ids.long()] + wd[top])).all())
    some = torch.zeros(v, dtype=torch.bool, device="cuda")
    some[ids.long()] = some[top] = True
    assert not bool(dw[~some].any())
