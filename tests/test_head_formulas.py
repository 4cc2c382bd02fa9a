"""The head's definitions in 64 bits: against the rows' definitions, and their gradients against differences."""
import numpy as np
import pytest
import torch

import util_head as uh
import util_rows as ur


def case(n=5, v=23, h=7, seed=1):
    x, w, ids, beta = uh.operands(n, v, h, "f32", seed, device="cpu")
    return x.double(), w.double(), ids, beta.double()


def test_forward_is_the_rows_log_probability():
    x, w, ids, beta = case()
    got, _ = uh.forward(x, w, ids, beta)
    want = ur.logprobs((x @ w.T).numpy(), ids.numpy(), beta.numpy())
    for name in ("logprob", "lse", "stats"):
        assert np.allclose(got[name].numpy(), want[name], rtol=1e-12, atol=1e-12), name


@pytest.mark.parametrize("seed", range(4))
def test_gradients_against_differences(seed):
    x, w, ids, beta = case(seed=seed)
    gen = torch.Generator().manual_seed(seed)
    g, q = torch.randn(5, generator=gen, dtype=torch.float64), torch.randn(5, generator=gen, dtype=torch.float64)
    ids[1] = -1
    g0 = torch.where(ids >= 0, g, torch.zeros_like(g))

    def value(x, w):
        r, _ = uh.forward(x, w, ids, beta)
        return float((g0 * torch.nan_to_num(r["logprob"])).sum() + (q * r["lse"]).sum())

    stats = uh.forward(x, w, ids, beta)[0]["stats"]
    dx, dw, _, _ = uh.backward(x, w, ids, stats, g, q, beta)
    for t, grad in ((x, dx), (w, dw)):
        for at in [(0, 0), (1, 2), (4, 6), (int(ids[0]) % len(t), 3)]:
            step = 1e-5
            old = float(t[at])
            t[at] = old + step
            up = value(x, w)
            t[at] = old - step
            down = value(x, w)
            t[at] = old
            assert abs((up - down) / (2 * step) - float(grad[at])) < 1e-8 * (1 + abs(float(grad[at]))) + 1e-8


def test_rows_without_a_weight_add_nothing():
    x, w, ids, beta = case()
    stats = uh.forward(x, w, ids, beta)[0]["stats"]
    g = torch.ones(5, dtype=torch.float64)
    ids2, x2 = ids.clone(), x.clone()
    ids2[2], x2[2] = -1, float("nan")
    dx, dw, _, _ = uh.backward(x2, w, ids2, stats, g, None, beta)
    keep = [0, 1, 3, 4]
    dx2, dw2, _, _ = uh.backward(x[keep], w, ids[keep], stats[keep], g[keep], None, beta[keep])
    assert torch.equal(dx[2], torch.zeros(7, dtype=torch.float64)) and torch.allclose(dx[keep], dx2) and torch.allclose(dw, dw2)
