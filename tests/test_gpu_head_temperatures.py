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


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("h", [96, 100, 512, 1000])
@pytest.mark.parametrize("n", [1, 7, 16, 17, 33, 64, 65, 130, 300])
def test_the_logits_formed_again_are_the_forward_pass_own(n, h, name):
    """With the statistics of the forward pass on the same operands the largest logit is M to the last bit, however they are summed: at
    an inverse temperature of 2^60 its p is 1 and those of the others, units below it, 0."""
    v, beta = 700, 2.0 ** 60
    x, w, ids, _ = uh.operands(n, v, h, name, seed=5)
    top = (x.double() @ w.double().T).argmax(1)
    ids = torch.where(torch.arange(n, device="cuda") % 3 == 2, ids.long(), top).int()
    b, g = torch.full((n,), beta, device="cuda"), torch.ones(n, device="cuda")
    stats = tt.head_logprobs(v, x, w, ids, inv_temperature=b).stats
    assert not bool(stats[:, 1].any())
    dx, dw = tt.head_logprobs_backward(v, x, w, ids, stats, g, inv_temperature=b)
    want = beta * (w.double()[ids.long()] - w.double()[top])
    # one or two entries of dz, powers of two: a sum of two and its rounding
    assert bool(((dx.double() - want).abs() <= (2 * uh.HALF_STEP[name] + 4 * uh.U) * beta * (w.double()[ids.long()].abs() + w.double()[top].abs())).all())
    assert not bool(dx[ids == top].any())


@pytest.mark.parametrize("n", [1, 7, 16, 17, 64, 100])
def test_gradients_of_tokens_that_are_almost_certain(n):
    """1 - p from 1e-2 down: its error is that of the other tokens' exponents, as in the forward pass, not a rounding of the token's own
    logit over 1 - p."""
    v, h = 640, 256
    x, w, ids, beta = uh.operands(n, v, h, "f32", seed=2, lean=0.0)
    x = 0.5 * x + 21.0 * w[ids.long()] / (w[ids.long()] ** 2).sum(1, keepdim=True)
    g = torch.ones(n, device="cuda")
    got = tt.head_logprobs(v, x, w, ids, inv_temperature=beta)
    assert float(got.logprob.min()) > -1e-2
    dx, _ = tt.head_logprobs_backward(v, x, w, ids, got.stats, g, inv_temperature=beta)
    z, off = uh.logits(x, w, "f32")
    y = z * beta.double()[:, None]
    at = ids.long()[:, None]
    rest = torch.logsumexp(y.scatter(1, at, -float("inf")), 1) - y.gather(1, at)[:, 0]  # ln of the others' sum over the token's term
    total = torch.log1p(rest.exp())
    d = -torch.exp(y - y.gather(1, at) - total[:, None])
    d.scatter_(1, at, -torch.expm1(-total)[:, None])
    d = d * beta.double()[:, None]
    wd = w.double()
    # an exponent is a difference of two logits, in the statistics and here; sums of 300 and 640 terms
    rel = 4 * beta.double()[:, None] * off[:, None] + uh.U * (300 + 640 + 100)
    assert bool(((dx.double() - d @ wd).abs() <= rel * (d.abs() @ wd.abs())).all())


@pytest.mark.parametrize("rows", [None, "64 bits", 1, 100])
@pytest.mark.parametrize("n", [1, 7, 16, 17, 64, 100, 300])
def test_statistics_of_another_product(n, rows):
    """In 64 bits and rounded, or from calls of other numbers of rows: their M is not the largest logit's sum here to the last bit.  1 - p from 1e-2 down: its error is that of the other tokens' exponents, as in the forward pass, not a rounding of the token's own
    logit over 1 - p."""
    v, h = 640, 256
    x, w, ids, beta = uh.operands(n, v, h, "f32", seed=2, lean=0.0)
    x = 0.5 * x + 21.0 * w[ids.long()] / (w[ids.long()] ** 2).sum(1, keepdim=True)
    g = torch.ones(n, device="cuda")
    got = tt.head_logprobs(v, x, w, ids, inv_temperature=beta)
    assert float(got.logprob.min()) > -1e-2
    stats = got.stats
    if rows == "64 bits":
        stats = uh.forward(x, w, ids, beta)[0]["stats"].float()
    elif rows:
        stats = torch.cat([tt.head_logprobs(v, x[i:i + rows].repeat(max(1, rows // len(x)) + 1, 1)[:rows], w).stats[:len(x[i:i + rows])] for i in range(0, n, rows)])
        stats[:, 1] = got.stats[:, 1]  # M does not depend on the temperatures
    dx, _ = tt.head_logprobs_backward(v, x, w, ids, stats, g, inv_temperature=beta)
    z, off = uh.logits(x, w, "f32")
    y = z * beta.double()[:, None]
    at = ids.long()[:, None]
    rest = torch.logsumexp(y.scatter(1, at, -float("inf")), 1) - y.gather(1, at)[:, 0]  # ln of the others' sum over the token's term
    total = torch.log1p(rest.exp())
    d = -torch.exp(y - y.gather(1, at) - total[:, None])
    d.scatter_(1, at, -torch.expm1(-total)[:, None])
    d = d * beta.double()[:, None]
    wd = w.double()
    # an exponent is a difference of two logits, in the statistics and here; sums of 300 and 640 terms
    rel = 4 * beta.double()[:, None] * off[:, None] + uh.U * (300 + 640 + 100)
    assert bool(((dx.double() - d @ wd).abs() <= rel * (d.abs() @ wd.abs())).all())


@pytest.mark.parametrize("n", [1, 8, 20, 64, 70, 300])
@pytest.mark.parametrize("gap,beta", [(2.0 ** -16, 1.0), (2.0 ** -16, 2.0 ** 12), (2.0 ** -16, 2.0 ** 18), (2.0 ** -16, 2.0 ** 20), (2.0 ** -19, 2.0 ** 24), (2.0 ** -4, 1.0), (0.25, 1.0)])
@pytest.mark.parametrize("own", [0, 1])
def test_two_tokens_side_by_side(own, gap, beta, n):
    """The largest logit and one a gap below it, without rounding errors: each keeps its own probability, near ties and at any
    temperature, whichever of them is the row's token."""
    v, h, a, t = 500, 64, 130, 7
    values = torch.full((v,), -200.0, dtype=torch.float64)
    values[a], values[t] = 16.0, 16.0 - gap
    w, x = torch.zeros((v, h), device="cuda"), torch.zeros((n, h), device="cuda")
    w[:, 3], x[:, 3] = values.float().cuda(), 1.0
    ids = torch.full((n,), (a, t)[own], dtype=torch.int32, device="cuda")
    b, g = torch.full((n,), beta, device="cuda"), torch.ones(n, device="cuda")
    stats = tt.head_logprobs(v, x, w, ids, inv_temperature=b).stats
    _, dw = tt.head_logprobs_backward(v, x, w, ids, stats, g, inv_temperature=b)
    q = torch.sigmoid(torch.tensor(-gap * beta, dtype=torch.float64))  # of the lower one, both ways as sigmoids
    d = torch.stack((q, -q) if own == 0 else (-torch.sigmoid(torch.tensor(gap * beta, dtype=torch.float64)), torch.sigmoid(torch.tensor(gap * beta, dtype=torch.float64)))) * beta * n
    got = dw[[a, t], 3].double().cpu()
    # exponents of up to 46 (base 2), three roundings each, in the statistics and here; 1 - p by the difference of an exponent and L, each
    # up to 1 where p is not small; n equal terms
    off = uh.U * (6 * 46 * 0.7 + 64 + n)
    assert bool(((got - d).abs() <= off * d.abs() + 2.0 ** -100 * beta).all()), (got, d)
