"""The gradients' formulas against central differences of the values' definitions, in 64 bits on the CPU."""
import numpy as np
import pytest

import util_rows as ur

H = 1e-5
# a central difference is off by H^2 / 6 of the third derivative (below 8 here, with weights up to 3) and by the
# values' rounding, 2^-53 of at most 64, over H
BOUND = 8 * 3 * H * H + 64 * 2.0 ** -53 / H


def differences(f, x):
    d = np.zeros_like(x)
    for j in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[j] += H
        down[j] -= H
        d[j] = (f(up) - f(down)) / (2 * H)
    return d


def test_logprobs_gradient():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((5, 13)) * 2
    x[1, 4] = -np.inf
    ids, beta = np.array([3, 5, -1, 0, 12]), 0.5 + rng.random(5)
    g, h = rng.standard_normal(5), rng.standard_normal(5)

    def value(y):
        r = ur.logprobs(y, ids, beta)
        return (np.where(ids >= 0, g * r["logprob"], 0.0) + h * r["entropy"]).sum()

    with np.errstate(invalid="ignore"):
        want = differences(value, x)
    got, _ = ur.logprobs_gradient(x, ids, beta, g, h)
    assert np.all(np.abs(got - want) <= BOUND)


@pytest.mark.parametrize("tail", [False, True])
def test_distill_gradient(tail):
    rng = np.random.default_rng(2)
    n, v, k = 6, 11, 5
    x = rng.standard_normal((n, v)) * 2
    ids = np.stack([rng.permutation(v)[:k] for _ in range(n)])
    lp = np.log(rng.dirichlet(np.ones(k), n) * 0.8)
    ids[1, 2] = ids[1, 0]
    ids[2, 1:] = -1
    lp[3, 0] = -np.inf
    ids[4] = -1
    x[5, [j for j in range(v) if j not in ids[5]][0]] = -np.inf
    beta, w = 0.5 + rng.random(n), rng.standard_normal(n)
    value = lambda y: (w * ur.distill(y, beta, ids, lp, tail)[0]).sum()  # noqa: E731
    with np.errstate(invalid="ignore"):
        want = differences(value, x)
    _, got, _, _ = ur.distill(x, beta, ids, lp, tail, weight=w)
    assert np.all(np.abs(got - want) <= BOUND)
    assert not got[4].any()
