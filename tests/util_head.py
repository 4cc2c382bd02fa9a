"""The operators on the output head in 64 bits (torch, CPU or GPU), from their definitions, with bounds on how far results
in the kernels' arithmetic may be from them, and inputs for their tests."""
import math

import torch

U = 2.0 ** -24  # half a step of fp32, relative to the value
HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}  # half of finfo(type).eps
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
# A gradient row's values as the products take them, at the scale of the largest row weight: relative and absolute rounding
# (fp16 is stored 2^14 times as large, so steps of 2^-24 are 2^-38)
STORED = {"bf16": (2.0 ** -8, 2.0 ** -126), "f16": (2.0 ** -11, 2.0 ** -39), "f32": (2.0 ** -23, 2.0 ** -120)}
LEAST = 2.0 ** -126  # fp32's (and bf16's) smallest normal value: what is smaller may count as 0, probabilities and results alike


def sum_error(terms, passes=1):
    """A sum of `terms` products in fp32 in any order, relative to the sum of their sizes: a rounding each, of at most a
    step (the matrix cores need not round to nearest); fp32 operands: of six products' sums, and what they leave out."""
    return 2 * U * (terms * passes + 16) + (2.0 ** -22 if passes > 1 else 0.0)


def passes(name):
    return 6 if name == "f32" else 1


def logits(x, w, name="f64"):
    """(z, a bound on the kernels' error of each row's logits) in 64 bits."""
    x, w = x.double(), w.double()
    z = x @ w.T
    size = (x.abs() @ w.abs().T).amax(1) if name != "f64" else z.new_zeros(len(x))
    return z, size * (sum_error(x.shape[1], passes(name)) if name != "f64" else 0.0)


def forward(x, w, ids=None, beta=None, name="f64"):
    """(logprob, lse, stats), and bounds for each."""
    z, off = logits(x, w, name)
    n, v = z.shape
    b = torch.ones(n, dtype=torch.float64, device=z.device) if beta is None else beta.double()
    m = z.amax(1)
    y = (z - m[:, None]) * b[:, None]
    log_sum = y.exp().sum(1).log()
    lse = b * m + log_sum
    logprob = None
    if ids is not None:
        logprob = (y.gather(1, ids.long().clamp(0, v - 1)[:, None])[:, 0] - log_sum)
        logprob = torch.where((ids >= 0) & (ids < v), logprob, torch.full_like(logprob, math.nan))
    # a tile's sum: chains of up to 256 terms and joins; exponents in base 2, 3 roundings each, weighted by their
    # probabilities: at most 6 ln v of them; the exponential and the logarithm, 2 steps each
    sums = U * (300 + 12 * math.log(v + 1) + 8)
    offs = {"stats": torch.stack((off + U * m.abs(), 2 * b * off + sums + U * log_sum.abs()), 1),
            "lse": b * off + sums + 2 * U * (lse.abs() + (b * m).abs() + log_sum.abs()), "logprob": None}
    if ids is not None:
        offs["logprob"] = 2 * b * off + sums + 4 * U * (logprob.abs() + log_sum.abs())
    return dict(logprob=logprob, lse=lse, stats=torch.stack((m, log_sum), 1)), offs


def backward(x, w, ids, stats, g, grad_lse=None, beta=None, name="f64"):
    """(dhidden, dweight), and bounds for both: stats are taken as given."""
    z, off = logits(x, w, name)
    x, w = x.double(), w.double()
    n, v = z.shape
    dev = z.device
    b = torch.ones(n, dtype=torch.float64, device=dev) if beta is None else beta.double()
    q = torch.zeros(n, dtype=torch.float64, device=dev) if grad_lse is None else grad_lse.double()
    if ids is None:
        ids, g = torch.full((n,), -1, device=dev), torch.zeros(n, dtype=torch.float64, device=dev)
    inside = (ids >= 0) & (ids < v)
    g = torch.where(inside, g.double(), torch.zeros_like(q))
    some = (g != 0) | (q != 0)
    m, log_sum = stats[:, 0].double(), stats[:, 1].double()
    lp = (z - m[:, None]) * b[:, None] - log_sum[:, None]
    p = lp.exp()
    d = (q - g)[:, None] * p
    # p: its logit's error, three roundings of the exponent (in base 2) and of what it is a difference of, the exponential's
    rel = (b * off)[:, None] * 1.01 + U * (4 * lp.abs() + 4 * log_sum.abs()[:, None] + 16)
    err = (q.abs() + g.abs())[:, None] * (rel * p + LEAST)
    at = ids.long().clamp(0, v - 1)[:, None]
    lt = lp.gather(1, at)
    own = g[:, None] * -torch.expm1(lt) + q[:, None] * lt.exp()
    own_err = rel.gather(1, at) * (g.abs() + q.abs())[:, None] * lt.exp() + 16 * U * (g[:, None] * torch.expm1(lt)).abs()
    d.scatter_(1, at, torch.where(inside[:, None], own, d.gather(1, at)))
    err.scatter_(1, at, torch.where(inside[:, None], own_err, err.gather(1, at)))
    d, err = d * b[:, None], err * b[:, None]
    d[~some], err[~some] = 0.0, 0.0
    x = torch.where(some[:, None], x, torch.zeros_like(x))
    if name == "f64":
        return d @ w, d.T @ x, None, None
    top = float((b * (g.abs() + q.abs()))[some].max()) if bool(some.any()) else 1.0
    step, least = STORED[name]
    err = err + (step + 4 * U) * d.abs() + least * top
    err[~some] = 0.0
    k = passes(name)
    dx, dw, size = d @ w, d.T @ x, d.abs() + err
    # splits of the vocabulary are summed beside each other
    dx_off = err @ w.abs() + sum_error(v, k) * (size @ w.abs()) + (HALF_STEP[name] + 16 * U) * dx.abs()
    dw_off = err.T @ x.abs() + sum_error(n, k) * (size.T @ x.abs()) + (HALF_STEP[name] + 2 * U) * dw.abs()
    dx_off, dw_off = dx_off + LEAST, dw_off + LEAST
    if name == "f16":  # results below the type's normal range round in steps of 2^-24
        dx_off, dw_off = dx_off + 2.0 ** -25, dw_off + 2.0 ** -25
    return dx, dw, dx_off, dw_off


# ------------------------------------------------------------------------------- inputs
def operands(n, v, h, name, seed=0, device="cuda", lean=8.0):
    """(hidden, weight, ids, inverse temperatures): logits of a few units, the tokens likely ones."""
    gen = torch.Generator(device="cpu").manual_seed(seed * 1000003 + n * 10007 + v * 101 + h)
    weight = torch.randn((v, h), generator=gen) / math.sqrt(h)
    ids = torch.randint(0, v, (n,), generator=gen)
    hidden = 2.0 * torch.randn((n, h), generator=gen) + lean * torch.rand((n, 1), generator=gen) * weight[ids]
    beta = 0.7 + 0.8 * torch.rand(n, generator=gen)
    return hidden.to(TYPES[name]).to(device), weight.to(TYPES[name]).to(device), ids.int().to(device), beta.to(device)


def placed(x, pad=0, shift=0, fill=float("nan")):
    """x in rows `pad` elements further apart, the first `shift` elements into its memory; `fill` between rows."""
    n, h = x.shape
    ld = h + pad
    flat = torch.full((shift + n * ld + 64,), fill, dtype=torch.float32, device=x.device).to(x.dtype)
    rows = flat[shift:shift + n * ld].view(n, ld)[:, :h]
    rows.copy_(x)
    return rows
