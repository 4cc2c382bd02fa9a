"""The operators on rows of logits in numpy and 64 bits, from their definitions, and inputs for their tests."""
import math

import numpy as np

U = 2.0 ** -24  # half a step of fp32, relative to the value
HALF_STEP = {"bf16": 2.0 ** -9 * 2, "f16": 2.0 ** -11, "f32": 2.0 ** -24}  # half of finfo(type).eps
SMALLEST = {"bf16": 2.0 ** -126, "f16": 2.0 ** -25, "f32": 2.0 ** -126}  # results below flush, or round in steps of it


def clean(x):
    """fp64 logits, NaN as minus infinity."""
    x = np.asarray(x, np.float64)
    return np.where(np.isnan(x), -np.inf, x)


def row_statistics(x, beta):
    """(M, L, lp) of one row; None where the row has no distribution."""
    m = x.max()
    if m == np.inf or not (0.0 < beta <= 2.0 ** 100):
        return None
    if m == -np.inf:
        return m, 0.0, np.full(len(x), -np.inf)
    z = (x - m) * beta
    log_sum = math.log(np.exp(z).sum())
    return m, log_sum, z - log_sum


def logprobs(x, ids=None, beta=None, n_top=0):
    x = clean(x)
    n, v = x.shape
    out = dict(logprob=np.full(n, np.nan), lse=np.full(n, np.nan), stats=np.full((n, 2), np.nan), entropy=np.full(n, np.nan),
               top_ids=np.full((n, n_top), -1, np.int64), top_logprobs=np.full((n, n_top), np.nan))
    for i in range(n):
        b = 1.0 if beta is None else float(beta[i])
        s = row_statistics(x[i], b)
        if s is None:
            continue
        m, log_sum, lp = s
        out["stats"][i] = m, log_sum
        out["lse"][i] = m * b + log_sum
        p = np.exp(lp)
        out["entropy"][i] = -(p[p > 0] * lp[p > 0]).sum()
        if ids is not None and 0 <= ids[i] < v:
            out["logprob"][i] = lp[ids[i]]
        out["top_logprobs"][i] = -np.inf
        order = np.argsort(-x[i], kind="stable")[:n_top]
        order = order[x[i][order] > -np.inf]
        out["top_ids"][i, :len(order)] = order
        out["top_logprobs"][i, :len(order)] = lp[order]
    return out


def logprobs_gradient(x, ids, beta, g, h):
    """(gradient, bound on the terms' sizes times the steps that they may be off by)."""
    x = clean(x)
    n, v = x.shape
    d, off = np.zeros((n, v)), np.zeros((n, v))
    for i in range(n):
        b = 1.0 if beta is None else float(beta[i])
        gi = float(g[i]) if g is not None and 0 <= ids[i] < v else 0.0
        hi = float(h[i]) if h is not None else 0.0
        if gi == 0.0 and hi == 0.0:
            continue
        s = row_statistics(x[i], b)
        if s is None:
            d[i] = np.nan
            continue
        m, log_sum, lp = s
        if m == -np.inf:
            continue
        p = np.exp(lp)
        lp0 = np.where(p > 0, lp, 0.0)
        entropy = -(p * lp0).sum()
        d[i] = -b * (gi * p + hi * p * (lp0 + entropy))
        # p: 3 roundings in its exponent's product and 1 of each of L and the difference, relative to the exponent,
        # 2 steps of the exponential; then products and sums of 4 terms
        steps = 4 * np.abs(lp0) + 2 * log_sum + 16
        off[i] = U * steps * b * (abs(gi) * p + abs(hi) * p * (np.abs(lp0) + entropy + 1))
        if gi != 0.0:
            t = ids[i]
            d[i, t] = b * (gi * -np.expm1(lp[t]) - hi * p[t] * (lp0[t] + entropy))
            # 1 - p from lp: lp is off by 4 steps of its size and of L's
            off[i, t] += U * b * abs(gi) * (16 * -np.expm1(lp[t]) + p[t] * (4 * abs(lp0[t]) + 4 * log_sum))
    return d, off


def distill_row(x, b, ids, a, tail):
    """(loss, gradient for weight 1, bound on the loss's error, on the gradient's) of one row; ids are the student's."""
    v = len(x)
    zeros = np.zeros(v)
    kept = [(int(t), float(c)) for t, c in zip(ids, a) if 0 <= t < v and c > -np.inf]
    s = row_statistics(x, b)
    if s is None or any(c == np.inf for _, c in kept):
        return np.nan, np.full(v, np.nan), 0.0, zeros
    m, log_sum, lp = s
    if not kept or m == -np.inf:
        return 0.0, zeros, 0.0, zeros
    if tail:
        weights = [math.exp(c) for _, c in kept]
    else:
        top = max(c for _, c in kept)
        weights = [math.exp(c - top) for _, c in kept]
        total = sum(weights)
        weights = [w / total for w in weights]
    mass = {}
    for (t, _), w in zip(kept, weights):
        mass[t] = mass.get(t, 0.0) + w
    unlisted = np.ones(v, bool)
    unlisted[list(mass)] = False
    open_ = unlisted & (x > -np.inf)
    listed = sum(mass.values())
    r = max(0.0, 1.0 - listed) if tail and open_.any() else 0.0
    q = np.exp(lp)
    loss, size = 0.0, 0.0
    for t, w in mass.items():
        if w > 0.0:
            loss += w * (math.log(w) - lp[t])
            size += w * (1.0 + (abs(lp[t]) if lp[t] > -np.inf else 0.0) + log_sum)
    d = (listed + r) * q
    share = 0.0
    if open_.any():
        top = x[open_].max()
        e = np.exp((x[open_] - top) * b)
        log_share = (top - m) * b + math.log(e.sum()) - log_sum
        share = math.exp(log_share)
        if r > 0.0:
            loss += r * (math.log(r) - log_share)
            size += r * (1.0 + abs(log_share) + log_sum)
        d[open_] = ((listed + r) * share - r) * (e / e.sum())
    for t, w in mass.items():
        d[t] = (listed + r) * q[t] - w
    # the unlisted sum is formed in fp32: a chain of at most 64 elements, each off by 3 steps of its exponent and 2 of
    # the exponential's, then a tree of 8 joins; the rest is fp64
    sums = U * (64 + 8 + 3 * 40)
    lp0 = np.where(q > 0, lp, 0.0)
    grad_off = np.abs(d) * U * (4 * np.abs(lp0) + 4 * log_sum + 16) + sums * (listed + r) * q
    return loss, d, sums * (listed + r) + U * size, grad_off


def distill(x, beta, top_ids, top_logprobs, tail, id_map=None, weight=None):
    x = clean(x)
    n, v = x.shape
    loss, d, loss_off, off = np.zeros(n), np.zeros((n, v)), np.zeros(n), np.zeros((n, v))
    for i in range(n):
        ids = np.asarray(top_ids[i], np.int64)
        if id_map is not None:
            ids = np.array([id_map[t] if 0 <= t < len(id_map) else -1 for t in ids], np.int64)
        b = 1.0 if beta is None else float(beta[i])
        loss[i], g, loss_off[i], o = distill_row(x[i], b, ids, np.asarray(top_logprobs[i], np.float64), tail)
        w = 1.0 if weight is None else float(weight[i])
        d[i] = 0.0 if w == 0.0 else w * b * g
        off[i] = abs(w) * b * o if w != 0.0 and 0.0 < b <= 2.0 ** 100 else 0.0
    return loss, d, loss_off, off


# ------------------------------------------------------------------------------- inputs on the GPU
def torch_type(name):
    import torch

    return {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[name]


def placed(x, dtype, pad=0, shift=0):
    """x (host fp32) as rows of `dtype` on the GPU, `pad` more elements to a row's stride, the first row `shift`
    elements into its memory; what lies between rows is NaN."""
    import torch

    n, v = x.shape
    ld = v + pad
    flat = torch.full((shift + n * ld + 64,), float("nan"), dtype=torch_type(dtype), device="cuda")
    rows = flat[shift:shift + n * ld].view(n, ld)[:, :v] if n else flat.view(1, -1)[:0, :v]
    rows.copy_(torch.from_numpy(np.ascontiguousarray(x, np.float32)))
    return rows


def host(t):
    return t.detach().double().cpu().numpy()


def model_rows(rng, n, v, spread=2.0):
    """Logits of a language model's shape: a wide bulk and some tokens that stand out."""
    x = (rng.standard_normal((n, v)) * spread).astype(np.float32)
    for i in range(n):
        at = rng.integers(0, v, 1 + v // 64 if v < 1024 else 24)
        x[i, at] = 3.0 + 9.0 * rng.random(len(at)) ** 2
    return x
