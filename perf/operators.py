"""Performance cases of the operators on logit rows: log probabilities, their gradient, distillation.

A case is a dict of plain values.  Its "kind" names the public call it stands for:

  logprobs    log probabilities of given tokens, log-sum-exp, entropy, top alternatives (tt.logprobs)
  backward    the gradient of log probabilities and entropies (tt.logprobs_backward)
  loss        the distillation loss of a teacher's top tokens (tt.distill)
  distill     the loss and its gradient in one call (tt.distill with grad_loss)

run() takes the framework's calls where `own` is true and otherwise the same operators in elementary torch
operations in fp32.  prepare() makes what a program has in hand: logits as the model's last product leaves them,
tokens, temperatures, the teacher's lists, upstream gradients, the saved statistics of the forward pass, and
buffers for large gradients.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f16": 2, "f32": 4}
_LARGEST = 1.2e9  # bytes that a drawn case moves at most


def listed():
    return [
        # one interactive stream of small models returns its token's log probability: launches are all there is
        dict(name="logprobs 1x640", kind="logprobs", n=1, v=640, dtype="bf16", top=5, entropy=False),
        # one stream of a large vocabulary, a decode step with alternatives
        dict(name="logprobs 1x151936 top20", kind="logprobs", n=1, v=151936, dtype="bf16", top=20, entropy=True),
        # a server's decode step, some of its rows held to a grammar
        dict(name="logprobs 48x128256 top8", kind="logprobs", n=48, v=128256, dtype="bf16", top=8, entropy=True, masked=0.2),
        # fp32 logits of an odd width, ragged batch of scored answers
        dict(name="logprobs 333x50257 f32", kind="logprobs", n=333, v=50257, dtype="f32", top=5, entropy=False),
        # a prompt's tokens scored, nothing else wanted
        dict(name="logprobs 4096x151936", kind="logprobs", n=4096, v=151936, dtype="bf16", top=0, entropy=False),
        # a teacher's lists for distillation, the largest vocabulary
        dict(name="logprobs 1024x262144 top64", kind="logprobs", n=1024, v=262144, dtype="bf16", top=64, entropy=False),
        # policy gradient with an entropy bonus
        dict(name="backward 2048x128256", kind="backward", n=2048, v=128256, dtype="bf16", entropy=True),
        # cross entropy of a ragged batch, odd width, fp16
        dict(name="backward 391x50257 f16", kind="backward", n=391, v=50257, dtype="f16", entropy=False),
        # validation of a drafter against its target's lists
        dict(name="loss 512x151936 top64", kind="loss", n=512, v=151936, dtype="bf16", top=64, tail=True),
        # a small drafter of another vocabulary on one accumulation step, fp32
        dict(name="distill 96x32000 f32 map", kind="distill", n=96, v=32000, dtype="f32", top=32, tail=False, v_map=50257, share=0.6),
        # a few rows only
        dict(name="distill 8x50257 top20", kind="distill", n=8, v=50257, dtype="bf16", top=20, tail=True),
        # the training step's rows
        dict(name="distill 2048x151936 top64", kind="distill", n=2048, v=151936, dtype="bf16", top=64, tail=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("logprobs", "logprobs", "backward", "loss", "distill", "distill"))
    v, dtype = _log_int(rng, 500, 262144), rng.choice(("bf16", "bf16", "f16", "f32"))
    passes = 2 if kind in ("backward", "distill") else 1
    n = _log_int(rng, 1, max(1, min(4096, int(_LARGEST / (passes * v * _BYTES[dtype])))))
    case = dict(kind=kind, n=n, v=v, dtype=dtype)
    if kind == "logprobs":
        return dict(case, top=rng.choice((0, 1, 5, 20, 64, 128)), entropy=rng.random() < 0.5, masked=rng.choice((0.0, 0.0, 0.3)))
    if kind == "backward":
        return dict(case, entropy=rng.random() < 0.5)
    case = dict(case, top=rng.choice((1, 8, 20, 50, 64, 128)), tail=rng.random() < 0.5)
    return dict(case, v_map=_log_int(rng, 2000, 262144), share=rng.choice((0.3, 0.8))) if rng.random() < 0.4 else case


# ------------------------------------------------------------------------------- inputs
def _rand(gen, *shape):
    return torch.rand(shape, generator=gen, device="cuda")


def _randint(gen, hi, *shape):
    return torch.randint(0, hi, shape, generator=gen, device="cuda")


def _distinct(gen, n, width, k):
    """k different tokens for each of n rows."""
    step = 1 + (_rand(gen, n, 1) * (width // k - 1)).long()
    return (_randint(gen, width, n, 1) + step * torch.arange(k, device="cuda")) % width


def _rows(case, gen):
    """fp32 logits of a language model's shape: a wide bulk and some tokens that stand out of it."""
    n, v = case["n"], case["v"]
    x = torch.randn((n, v), generator=gen, device="cuda") * 2.0
    at = _distinct(gen, n, v, 24)
    return x.scatter_(1, at, 3.0 + 9.0 * _rand(gen, n, 24) ** 2), at


def _statistics(logits, beta):
    """What a forward pass saved: the largest logit, the log of the sum relative to it, the entropy."""
    stats = torch.empty((logits.shape[0], 2), device="cuda")
    entropy = torch.empty(logits.shape[0], device="cuda")
    for a in range(0, logits.shape[0], 256):
        x = logits[a:a + 256].double()
        m = x.amax(1, keepdim=True)
        z = (x - m) * beta[a:a + 256, None].double()
        log_sum = z.exp().sum(1, keepdim=True).log()
        lp = z - log_sum
        stats[a:a + 256, :1], stats[a:a + 256, 1:] = m, log_sum
        entropy[a:a + 256] = -torch.where(lp > -1e4, lp.exp() * lp, torch.zeros_like(lp)).sum(1)
    return stats, entropy


def _teacher(case, gen, logits):
    """The teacher's lists (ids, log probabilities) and the map to the student's vocabulary, if that is another
    one; the student's logits are raised where the teacher's are high, so that the two nearly agree."""
    n, v, k = case["n"], case["v"], case["top"]
    width = case.get("v_map", v)
    k = min(k, width)
    ids = _distinct(gen, n, width, k)
    raw = -1.2 * torch.log1p(torch.arange(k, device="cuda", dtype=torch.float32)) + 0.3 * torch.randn((n, k), generator=gen, device="cuda")
    raw = raw.sort(1, descending=True).values
    logprobs = raw - raw.logsumexp(1, keepdim=True) + torch.log(0.6 + 0.38 * _rand(gen, n, 1))
    id_map, mapped = None, ids
    if "v_map" in case:
        shared = max(1, int(case["share"] * min(v, width)))
        id_map = torch.full((width,), -1, dtype=torch.int32, device="cuda")
        id_map[torch.randperm(width, generator=gen, device="cuda")[:shared]] = torch.randperm(v, generator=gen, device="cuda")[:shared].int()
        mapped = id_map[ids].long()
    raised = 12.0 + logprobs + 0.5 * torch.randn((n, k), generator=gen, device="cuda")
    row = torch.arange(n, device="cuda")[:, None].expand(n, k)
    keep = mapped >= 0
    logits[row[keep], mapped[keep]] = raised[keep]
    return ids.int(), logprobs, id_map


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 4 + 1)
    n, v, dtype = case["n"], case["v"], _DTYPES[case["dtype"]]
    x, at = _rows(case, gen)
    state = dict(case, beta=0.7 + 0.8 * _rand(gen, n))
    if case["kind"] in ("logprobs", "backward"):
        ids = torch.where(_rand(gen, n) < 0.7, at[:, 0], _randint(gen, v, n))
        held = int(math.ceil(case.get("masked", 0.0) * n))  # rows that a grammar holds to a few tokens
        if held:
            x[:held][_rand(gen, held, v) > 0.02] = -math.inf
            x[torch.arange(held, device="cuda"), ids[:held]] = 3.0
        state.update(logits=x.to(dtype), ids=ids.int())
    else:
        ids, logprobs, id_map = _teacher(case, gen, x)
        state.update(logits=x.to(dtype), ids=ids, logprobs=logprobs, id_map=id_map)
    if case["kind"] == "backward":
        state["stats"], state["h"] = _statistics(state["logits"], state["beta"])
        state.update(g=torch.randn(n, generator=gen, device="cuda") / n, gh=0.01 * (0.5 + _rand(gen, n)) / n)
    if case["kind"] == "distill":
        state["g"] = (0.5 + _rand(gen, n)) / n
    if case["kind"] in ("backward", "distill"):
        state["g"] = state["g"] * (1024.0 if case["dtype"] == "f16" else 1.0)  # the loss scale of fp16 training
        state["out"] = torch.empty_like(state["logits"])
    return state


# ------------------------------------------------------------------------------- the framework's calls
def _own(s):
    import paper_2510_15545_amd as tt

    kind, v = s["kind"], s["v"]
    if kind == "logprobs":
        r = tt.logprobs(v, s["logits"], s["ids"], inv_temperature=s["beta"], n_top=s["top"], entropy=s["entropy"])
        return r._asdict()
    if kind == "backward":
        more = dict(entropy=s["h"], grad_entropy=s["gh"]) if s["entropy"] else {}
        return {"dlogits": tt.logprobs_backward(v, s["logits"], s["ids"], s["stats"], s["g"], inv_temperature=s["beta"], out=s["out"], **more)}
    more = dict(grad_loss=s["g"], dlogits=s["out"]) if kind == "distill" else {}
    loss, grad = tt.distill(v, s["logits"], s["ids"], s["logprobs"], tail=s["tail"], id_map=s["id_map"], inv_temperature=s["beta"], **more)
    return {"loss": loss, "dlogits": grad}


# ------------------------------------------------------------------------------- the plain forms
def _order_keys(x):
    """int64 keys of fp32 values: larger value first, then the lower index; the lowest key for -inf."""
    bits = (x + 0.0).view(torch.int32)
    bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    index = torch.arange(x.shape[1], device=x.device)
    return (bits << 32) + (0x7FFFFFFF - index)


def _plain_logprobs(s):
    x = s["logits"].float()
    n, v = x.shape
    top_x = x.amax(1, keepdim=True)
    z = (x - top_x) * s["beta"][:, None]
    e = z.exp()
    log_sum = e.sum(1, keepdim=True).log()
    lse = top_x * s["beta"][:, None] + log_sum
    out = {"logprob": (z.gather(1, s["ids"].long()[:, None]) - log_sum)[:, 0], "lse": lse[:, 0], "stats": torch.cat((top_x, log_sum), 1),
           "entropy": None, "top_ids": None, "top_logprobs": None}
    if s["entropy"]:
        out["entropy"] = log_sum[:, 0] - torch.where(e > 0, e * z, torch.zeros_like(z)).sum(1) / e.sum(1)
    if s["top"]:
        at = _order_keys(x).topk(s["top"], 1).indices
        values = x.gather(1, at)
        lp = (values - top_x) * s["beta"][:, None] - log_sum
        out["top_ids"] = torch.where(values > -math.inf, at, torch.full_like(at, -1)).int()
        out["top_logprobs"] = torch.where(values > -math.inf, lp, torch.full_like(lp, -math.inf))
    return out


def _plain_backward(s):
    beta = s["beta"][:, None]
    lp = (s["logits"].float() - s["stats"][:, :1]) * beta - s["stats"][:, 1:]
    p = lp.exp()
    g = s["g"][:, None]
    d = -g * p
    if s["entropy"]:
        d = d - s["gh"][:, None] * p * (lp + s["h"][:, None])
    at = s["ids"].long()[:, None]
    d.scatter_(1, at, d.gather(1, at) + g * p.gather(1, at) - g * torch.expm1(lp.gather(1, at)))
    return {"dlogits": (d * beta).to(s["logits"].dtype)}


def _plain_distill(s):
    x = s["logits"].float()
    n, v = x.shape
    ids = s["ids"].long() if s["id_map"] is None else s["id_map"][s["ids"].long()].long()
    a = s["logprobs"].double()
    keep = (ids >= 0) & (ids < v) & (a > -math.inf)
    w = torch.where(keep, a.exp(), torch.zeros_like(a))
    if s["tail"]:
        rest = (1.0 - w.sum(1, keepdim=True)).clamp_min(0.0)
    else:
        w = w / w.sum(1, keepdim=True).clamp_min(1e-300)
        rest = torch.zeros_like(w[:, :1])
    at = torch.where(keep, ids, torch.full_like(ids, v))
    target = torch.zeros((n, v + 1), device=x.device).scatter_add_(1, at, w.float())[:, :v]
    listed_ = torch.zeros((n, v + 1), dtype=torch.bool, device=x.device).scatter_(1, at, True)[:, :v]
    z = (x - x.amax(1, keepdim=True)) * s["beta"][:, None]
    e = z.exp()
    total = e.sum(1, keepdim=True)
    outside = torch.where(listed_, torch.zeros_like(e), e).sum(1, keepdim=True)
    any_listed = keep.any(1, keepdim=True)
    r = torch.where((outside > 0) & any_listed, rest, torch.zeros_like(rest))
    log_q = z - total.log()
    # the terms nearly cancel where the two models agree: in 64 bits, by the lists' entries
    safe = torch.where(keep, ids, torch.zeros_like(ids))
    term = w * (target.gather(1, safe).double().log() - z.gather(1, safe).double() + total.double().log())
    loss = torch.where(w > 0, term, torch.zeros_like(term)).sum(1, keepdim=True)
    ratio = outside.double() / total.double()
    loss = loss + torch.where(r > 0, r * (r.log() - ratio.log()), torch.zeros_like(r))
    out = {"loss": loss[:, 0].float(), "dlogits": None}
    if s["kind"] == "distill":
        mass = w.sum(1, keepdim=True) + r
        factor = torch.where(r > 0, mass - r / ratio, mass).float()
        d = torch.where(listed_, mass.float() * log_q.exp() - target, factor * log_q.exp())
        out["dlogits"] = (d * (s["beta"] * s["g"])[:, None]).to(s["logits"].dtype)
    return out


def run(state):
    if own:
        return _own(state)
    if state["kind"] == "logprobs":
        return _plain_logprobs(state)
    return _plain_backward(state) if state["kind"] == "backward" else _plain_distill(state)


# ------------------------------------------------------------------------------- what a pass cannot do without
def work(case):
    n, v, e, k = case["n"], case["v"], _BYTES[case["dtype"]], case.get("top", 0)
    row = n * v * e
    if case["kind"] == "logprobs":  # the row; token, temperature; logprob, lse, statistics, entropy, list
        return {"bytes": row + n * (8 + 16 + (4 if case["entropy"] else 0) + 8 * k), "flops": n * v * (6 if case["entropy"] else 4)}
    if case["kind"] == "backward":
        return {"bytes": 2 * row + n * (8 + 8 + 4 + (8 if case["entropy"] else 0)), "flops": n * v * (7 if case["entropy"] else 4)}
    lists = n * (8 * k + 8) + (4 * n * k if "v_map" in case else 0)
    if case["kind"] == "loss":
        return {"bytes": row + lists, "flops": n * v * 4}
    return {"bytes": 2 * row + lists + 4 * n, "flops": n * v * 7}


# ------------------------------------------------------------------------------- 64 bits
def _exact_rows(x, beta):
    lse = torch.logsumexp(x * beta[:, None], 1)
    return lse, x * beta[:, None] - lse[:, None]


def exact(case, seed):
    s = prepare(case, seed)
    x, beta = s["logits"].double(), s["beta"].double()
    n, v = x.shape
    row = torch.arange(n, device=x.device)
    lse, lp = _exact_rows(x, beta)
    if case["kind"] == "logprobs":
        m = x.max(1).values
        out = {"logprob": lp[row, s["ids"].long()], "lse": lse, "stats": torch.stack((m, lse - beta * m), 1), "entropy": None, "top_ids": None, "top_logprobs": None}
        if case["entropy"]:
            out["entropy"] = torch.special.entr(lp.exp()).sum(1)
        if case["top"]:
            best = torch.full((n, case["top"]), -math.inf, dtype=torch.float64, device=x.device)
            values = x.sort(1, descending=True).values[:, :case["top"]]
            best[:, :values.shape[1]] = values * beta[:, None] - lse[:, None]
            out["top_logprobs"] = best
        return out
    if case["kind"] == "backward":
        p, hit = lp.exp(), torch.zeros_like(lp)
        hit[row, s["ids"].long()] = 1.0
        d = s["g"].double()[:, None] * (hit - p)
        if case["entropy"]:
            h = torch.special.entr(p).sum(1)
            d -= s["gh"].double()[:, None] * (p * lp.clamp_min(-1e30) + p * h[:, None])
        return {"dlogits": d * beta[:, None]}
    # the lists as lists: equal tokens of a row share one entry, the first of them
    ids = s["ids"].long() if s["id_map"] is None else s["id_map"].long()[s["ids"].long()]
    a = s["logprobs"].double()
    kept = (ids >= 0) & (ids < v)
    w = a.exp() * kept
    if not case["tail"]:
        w = w / w.sum(1, keepdim=True).clamp_min(1e-300)
    same = (ids[:, :, None] == ids[:, None, :]) & kept[:, :, None] & kept[:, None, :]
    first = kept & ~(same & torch.ones_like(same[0]).tril(-1)).any(2)
    mass = (same * w[:, None, :]).sum(2) * first
    at = ids.clamp(0, v - 1)
    lq = lp.gather(1, at)
    loss = (torch.special.xlogy(mass, mass) - mass * torch.where(first, lq, torch.zeros_like(lq))).sum(1)
    inside = x.scatter(1, torch.where(first, at, at[:, :1] * 0 + at), -math.inf) if bool(kept.all()) else None
    if inside is None:
        wide = torch.cat((x, torch.zeros_like(x[:, :1])), 1)
        inside = wide.scatter_(1, torch.where(kept, ids, torch.full_like(ids, v)), -math.inf)[:, :v]
    left = (torch.logsumexp(inside * beta[:, None], 1) - lse).exp()
    r = (1.0 - mass.sum(1)).clamp_min(0.0) * float(case["tail"]) * kept.any(1) * (left > 0)
    loss = loss + torch.where(r > 0, torch.special.xlogy(r, r / left), torch.zeros_like(r))
    if case["kind"] == "loss":
        return {"loss": loss, "dlogits": None}
    total = mass.sum(1) + r
    q = lp.exp()
    d = q * (total - torch.where(r > 0, r / left, torch.zeros_like(r)))[:, None]
    there = (total[:, None] * q.gather(1, at) - mass)[first]
    d[row[:, None].expand_as(ids)[first], at[first]] = there
    return {"loss": loss, "dlogits": d * (beta * s["g"].double())[:, None]}
