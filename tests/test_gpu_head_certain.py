"""Log probabilities of tokens that are almost certain, whose digits lie in what the other tokens leave, and of equally likely ones."""
import math

import pytest
import torch

import paper_2510_15545_amd as tt
import util_head as uh

pytestmark = pytest.mark.gpu

# rows and elements for each way of the product: few rows, a few, tiles, any alignment
WAYS = [(1, 64), (8, 64), (16, 65), (20, 64), (40, 65), (64, 64), (70, 64), (130, 128), (300, 64), (100, 33)]


def logits_at(n, h, values, name):
    """(hidden, weight) whose logits are exactly `values` [v], the same in every row: one element of each is not 0."""
    w = torch.zeros((len(values), h), device="cuda")
    w[:, 1] = torch.as_tensor(values, dtype=torch.float32)
    x = torch.zeros((n, h), device="cuda")
    x[:, 1] = 1.0
    return x.to(uh.TYPES[name]), w.to(uh.TYPES[name])


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,h", WAYS)
@pytest.mark.parametrize("v,top", [(640, 3), (2, 1), (1000, 999), (5003, 2500), (40001, 128)])
def test_an_almost_certain_token(v, top, n, h, name):
    """Logits without rounding errors, 8 to 31 below the largest one: L to the roundings of its own terms (3 each in the exponent, its
    sums' and joins', as in util_head), relative to itself and not to the 1 beside it."""
    values = -torch.randint(64, 256, (v,), generator=torch.Generator().manual_seed(v)).float() / 8
    values[top] = 0.0
    x, w = logits_at(n, h, values, name)
    ids = torch.full((n,), top, dtype=torch.int32, device="cuda")
    others = torch.cat((values[:top], values[top + 1:])).double()
    for beta in (1.0, 0.75):
        got = tt.head_logprobs(v, x, w, ids, inv_temperature=torch.full((n,), beta, device="cuda"))
        want = math.log1p(float((others * beta).exp().sum()))
        # an exponent of 46 (31 in base 2): 3 roundings of it, in 2^.; sums of up to 300 terms; the logarithm
        off = want * uh.U * (3 * 46 * math.log(2) + 300 + 16)
        assert float((got.stats[:, 1].double() - want).abs().max()) <= off
        assert float((got.logprob.double() + want).abs().max()) <= off
        assert float((got.lse.double() - want).abs().max()) <= off


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("n,h", WAYS)
@pytest.mark.parametrize("places", [(0, 1), (0, 4), (5, 21), (0, 64), (3, 131), (7, 300), (127, 128, 255, 256), (0, 699), tuple(range(700)), (2, 2 + 16, 2 + 32, 2 + 512)])
def test_equally_likely_tokens(places, n, h, name):
    """Largest logits that lie in one lane, wave, tile or in several: each counts once."""
    values = torch.full((700,), -40.0)
    values[list(places)] = 2.5
    x, w = logits_at(n, h, values, name)
    ids = torch.full((n,), places[-1], dtype=torch.int32, device="cuda")
    got = tt.head_logprobs(700, x, w, ids)
    want = math.log(len(places) + (700 - len(places)) * math.exp(-42.5))
    assert bool((got.stats[:, 0] == 2.5).all())
    assert float((got.stats[:, 1].double() - want).abs().max()) <= 4 * uh.U * want
    assert float((got.logprob.double() + want).abs().max()) <= 4 * uh.U * want


@pytest.mark.parametrize("n", [1, 8, 20, 70, 130])
@pytest.mark.parametrize("size", [10.0, 14.0])
def test_tokens_that_their_hidden_states_lean_towards(n, size):
    """As in a trained model's confident rows: relative errors of single log probabilities, under those of the logits' sums (twice,
    a difference) and of the sum of exponentials."""
    v, h = 640, 64
    x, w, ids, beta = uh.operands(n, v, h, "bf16", lean=0.0)
    x = (x.float() * 0.5 + size * w[ids.long()].float() / (w[ids.long()].float() ** 2).sum(1, keepdim=True) * 1.5).bfloat16()
    got = tt.head_logprobs(v, x, w, ids, inv_temperature=beta)
    want, _ = uh.forward(x, w, ids, beta)
    _, off = uh.logits(x, w, "bf16")
    rel = 2 * beta.double() * off + uh.U * (300 + 12 * math.log(v + 1) + 16)
    assert bool(((got.logprob.double() - want["logprob"]).abs() <= rel * want["logprob"].abs()).all())


@pytest.mark.parametrize("n", [1, 20, 100])
def test_the_gradient_of_an_almost_certain_token(n):
    """1 - p of a token that is almost certain: dhidden = beta g sum_j p_j (w_top - w_j), relative to its own size."""
    v, h = 640, 64
    values = -torch.randint(80, 160, (v,), generator=torch.Generator().manual_seed(1)).float() / 8
    values[5] = 0.0
    x, w = logits_at(n, h, values, "f32")
    ids = torch.full((n,), 5, dtype=torch.int32, device="cuda")
    g = torch.full((n,), 2.0, device="cuda")
    stats = tt.head_logprobs(v, x, w, ids).stats
    dx, dw = tt.head_logprobs_backward(v, x, w, ids, stats, g)
    p = torch.softmax(values.double().cuda(), 0)
    want = 2.0 * (p * -w.double()[:, 1]).sum()
    own = 2.0 * (p.sum() - p[5])
    # exponents as above; a sum of 640 positive terms
    off = uh.U * (3 * 31 * math.log(2) + 300 + 640 + 32)
    assert float((dx[:, 1].double() / want - 1).abs().max()) <= off
    assert float((dw[5, 1].double() / (n * own) - 1).abs().max()) <= off
