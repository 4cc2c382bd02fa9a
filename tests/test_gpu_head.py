"""tt_head_logprobs and tt_head_logprobs_backward against their definitions in 64 bits, within bounds derived from their
roundings: sizes of every kind, layouts, rows without a weight, rows without a distribution, graphs, streams."""
import math

import pytest
import torch

import paper_2510_15545_amd as tt
import util_head as uh

pytestmark = pytest.mark.gpu

NAN = float("nan")
SIZES = [(1, 1, 1), (1, 640, 256), (2, 2, 3), (3, 129, 65), (5, 1000, 1), (16, 513, 64), (17, 384, 72), (33, 300, 128), (64, 5000, 200),
         (9, 2100, 544), (16, 333, 1536), (12, 100, 4100), (65, 1025, 192), (400, 1500, 512), (130, 257, 64), (257, 513, 96), (300, 131, 1031), (1, 20011, 40), (129, 128, 2048), (600, 700, 33)]
LAYOUTS = [(0, 0), (8, 0), (3, 1)]  # of rows further apart, and of the first one off its alignment


def close(got, want, off, what):
    got = got.double()
    assert got.shape == want.shape, what
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    ok = torch.isnan(want) | (got == want) | ((got - want).abs() <= off)
    if not bool(ok.all()):
        at = (~ok).nonzero()[0].tolist()
        raise AssertionError(f"{what} at {at}: {float(got[tuple(at)])!r}, {float(want[tuple(at)])!r} +- {float(off[tuple(at)])!r}; {int((~ok).sum())} of {ok.numel()}")


def check_forward(v, x, w, ids, beta, name, **kw):
    got = tt.head_logprobs(v, x, w, ids, inv_temperature=beta, **kw)
    want, off = uh.forward(x, w[:v], ids, beta, name)
    for part in ("stats", "lse") + (("logprob",) if ids is not None else ()):
        close(getattr(got, part), want[part], off[part], part)
    return got


def check_backward(v, x, w, ids, stats, g, q, beta, name, **kw):
    dx, dw = tt.head_logprobs_backward(v, x, w, ids, stats, g, grad_lse=q, inv_temperature=beta, **kw)
    want_dx, want_dw, dx_off, dw_off = uh.backward(x, w[:v], ids, stats, g, q, beta, name)
    if dx is not None:
        close(dx[:len(x), :x.shape[1]], want_dx, dx_off, "dhidden")
    if dw is not None:
        close(dw[:v, :x.shape[1]], want_dw, dw_off, "dweight")
    return dx, dw


def weights(n, seed=0):
    gen = torch.Generator().manual_seed(seed + 77 * n)
    return (torch.rand(n, generator=gen) + 0.5).cuda(), torch.randn(n, generator=gen).cuda()


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,v,h", SIZES)
def test_sizes_and_layouts(n, v, h, name):
    x, w, ids, beta = uh.operands(n, v, h, name)
    g, q = weights(n)
    for pad, shift in LAYOUTS:
        print(f"[case] {n}x{v}x{h} {name} pad {pad} shift {shift}", flush=True)
        xs, ws = uh.placed(x, pad, shift), uh.placed(w, pad, shift)
        got = check_forward(v, xs, ws, ids, beta, name)
        check_backward(v, xs, ws, ids, got.stats, g, None, beta, name)
    print("[case] no temperatures, weights of the log-sum-exp too", flush=True)
    got = check_forward(v, x, w, ids, None, name)
    check_backward(v, x, w, ids, got.stats, -g, q, None, name)


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_fewer_tokens_than_the_weights_have(name):
    x, w, ids, beta = uh.operands(9, 500, 64, name)
    g, _ = weights(9)
    for v in (1, 130, 499):
        print(f"[case] {v} of 500", flush=True)
        inside = ids % v
        w2 = w.clone()
        w2[v:] = NAN
        got = check_forward(v, x, w2, inside.int(), beta, name)
        out = torch.full_like(w2, 7.0)
        check_backward(v, x, w2, inside.int(), got.stats, g, None, beta, name, dweight=out)
        assert bool((out[v:] == 7.0).all())


@pytest.mark.parametrize("name,v", [("bf16", 400003), ("f32", 120001)])
def test_pieces_of_a_large_vocabulary(name, v):
    x, w, ids, beta = uh.operands(3, v, 8, name, lean=14.0)
    ids[0], ids[1] = v - 1, 0
    g, q = weights(3)
    got = check_forward(v, x, w, ids, beta, name)
    check_backward(v, x, w, ids, got.stats, g, q, beta, name)


def test_large_and_small_values():
    """Logits of thousands, where only the largest counts, and of thousandths."""
    for name in ("bf16", "f16", "f32"):
        for scale in (300.0, 1e-3):
            print(f"[case] {name} x {scale}", flush=True)
            x, w, ids, beta = uh.operands(40, 700, 96, name)
            x = (x.float() * scale).to(x.dtype)
            g, q = weights(40)
            got = check_forward(700, x, w, ids, beta, name)
            check_backward(700, x, w, ids, got.stats, g, q, beta, name)


@pytest.mark.parametrize("sign", [-1.0, 1.0])
@pytest.mark.parametrize("n", [3, 20, 40, 100, 200])
@pytest.mark.parametrize("v,h", [(129, 64), (257, 64), (1000, 64), (1000, 63)])
def test_logits_all_far_from_zero(n, v, h, sign):
    """Sets without a logit (a tile's masked end) beside sums relative to a largest logit of minus two thousand."""
    x, w, ids, _ = uh.operands(n, v, h, "bf16")
    x[:, 0], w[:, 0] = sign * 100.0, 20.0
    g, _ = weights(n)
    got = check_forward(v, x, w, ids, None, "bf16")
    assert bool((got.stats[:, 0].abs() > 1900).all())
    check_backward(v, x, w, ids, got.stats, g, None, None, "bf16")


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
def test_rows_without_a_weight_are_not_read(name):
    n, v, h = 300, 450, 80
    x, w, ids, beta = uh.operands(n, v, h, name)
    g, _ = weights(n)
    stats = tt.head_logprobs(v, x, w, ids, inv_temperature=beta).stats
    gen = torch.Generator().manual_seed(3)
    for share in (0.0, 0.3, 0.9, 1.0):
        print(f"[case] {name} {share}", flush=True)
        out = (torch.rand(n, generator=gen) < share).cuda()
        ids2, g2, x2, stats2 = ids.clone(), g.clone(), x.clone(), stats.clone()
        ids2[out] = torch.where(torch.rand(n, generator=gen).cuda() < 0.5, -1, v)[out].int()
        x2[out], stats2[out] = NAN, NAN
        ids2[torch.nonzero(out)[:2]] = 5  # a token, and no weight
        g2[torch.nonzero(out)[:2]] = 0.0
        dx, dw = check_backward(v, x2, w, ids2, stats2, g2, None, beta, name)
        assert not bool(dx[out].any())
        if share == 1.0:
            assert not bool(dw.any())
    none = torch.zeros(n, device="cuda")
    dx, dw = tt.head_logprobs_backward(v, x2, w, None, stats2, None)
    assert not bool(dx.any()) and not bool(dw.any())
    dx, dw = tt.head_logprobs_backward(v, x2, w, ids, stats2, none, grad_lse=none)
    assert not bool(dx.any()) and not bool(dw.any())


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_weights_of_the_log_sum_exp_alone(name):
    x, w, ids, beta = uh.operands(70, 333, 48, name)
    _, q = weights(70)
    stats = tt.head_logprobs(333, x, w, inv_temperature=beta).stats
    check_backward(333, x, w, None, stats, None, q, beta, name)


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_row_weights_of_very_different_sizes(name):
    x, w, ids, beta = uh.operands(50, 300, 64, name)
    g = torch.logspace(-9, 3, 50).cuda()
    stats = tt.head_logprobs(300, x, w, ids, inv_temperature=beta).stats
    dx, _ = tt.head_logprobs_backward(300, x, w, ids, stats, g, inv_temperature=beta)
    for i in range(0, 50, 7):  # each row within its own weight's bounds
        want, _, off, _ = uh.backward(x[i:i + 1], w, ids[i:i + 1], stats[i:i + 1], g[i:i + 1], None, beta[i:i + 1], name)
        close(dx[i:i + 1], want, off, f"row {i}")


@pytest.mark.parametrize("name", ["bf16", "f16"])
@pytest.mark.parametrize("n,v,h", [(1, 640, 64), (1, 5000, 200), (3, 700, 64), (17, 300, 65), (64, 1000, 128)])
def test_few_rows_keep_what_rounding_takes(n, v, h, name):
    """Up to 64 rows: errors of the one rounding of the result (at most half a step of every value, and what the logits' sums are
    off), not of the logits' gradient's as well."""
    x, w, ids, beta = uh.operands(n, v, h, name)
    g, _ = weights(n)
    stats = tt.head_logprobs(v, x, w, ids, inv_temperature=beta).stats
    got = tt.head_logprobs_backward(v, x, w, ids, stats, g, inv_temperature=beta)
    want = uh.backward(x, w, ids, stats, g, None, beta, name)[:2]
    for a, b in zip(got, want):
        # errors uniform within half a step, which is at most HALF_STEP of the value: a mean square of at most HALF_STEP^2 / 3,
        # known to 0.9 / sqrt(N) of it for N equal values, N / 3 of normal ones: the root to four of 0.45 sqrt(3 / N)
        most = uh.HALF_STEP[name] * (3.0 ** -0.5 * (1 + 4 * 0.45 * (3 / b.numel()) ** 0.5) + 2.0 ** -5)
        assert float((a.double() - b).norm() / b.norm()) <= most


def test_one_gradient_alone():
    x, w, ids, beta = uh.operands(40, 300, 64, "bf16")
    g, _ = weights(40)
    stats = tt.head_logprobs(300, x, w, ids, inv_temperature=beta).stats
    both = tt.head_logprobs_backward(300, x, w, ids, stats, g, inv_temperature=beta)
    for want in (dict(dweight=False), dict(dhidden=None)):
        got = tt.head_logprobs_backward(300, x, w, ids, stats, g, inv_temperature=beta, **want)
        for a, b, name in zip(got, both, ("dhidden", "dweight")):
            assert a is None if name in want else torch.equal(a, b)


def test_rows_without_a_distribution():
    """NaN or infinite hidden states and temperatures outside (0, 2^100]: their rows are NaN, the others are not touched."""
    for name in ("bf16", "f16", "f32"):
        x, w, ids, beta = uh.operands(150, 260, 40, name)
        g, _ = weights(150)
        want = tt.head_logprobs(260, x, w, ids, inv_temperature=beta)
        bad = [3, 64, 90, 100, 127, 128, 149]
        x[3, 5], x[64, 39], x[90, 0] = NAN, float("inf"), -float("inf")
        beta[100], beta[127], beta[128], beta[149] = 0.0, -1.0, NAN, 2.0 ** 101
        got = tt.head_logprobs(260, x, w, ids, inv_temperature=beta)
        good = torch.ones(150, dtype=torch.bool)
        good[bad] = False
        for a, b in zip(got, want):
            assert bool(torch.isnan(a[~good]).all()) and torch.equal(a[good], b[good])
        dx, dw = tt.head_logprobs_backward(260, x, w, ids, got.stats, g, inv_temperature=beta)
        assert bool(torch.isnan(dx[~good]).all()) and not bool(torch.isnan(dx[good]).any()) and bool(torch.isnan(dw).all())
        keep = torch.nonzero(good)[:, 0].cuda()
        want_dx, _, off, _ = uh.backward(x[keep], w, ids[keep], got.stats[keep], g[keep], None, beta[keep], name)
        # the largest row weight is that of the sound rows
        close(dx[keep], want_dx, off, "dhidden")
        ids2 = ids.clone()
        ids2[bad] = -1  # without a weight they add nothing
        check_backward(260, torch.where(torch.isfinite(x), x, torch.zeros_like(x)), w, ids2, got.stats, g, None,
                       torch.where((beta > 0) & (beta < 9), beta, torch.ones_like(beta)), name)
        dx, dw = tt.head_logprobs_backward(260, x, w, ids2, got.stats, g, inv_temperature=beta)
        assert bool(torch.isfinite(dw.float()).all()) and not bool(dx[~good].any())


def test_logits_of_minus_infinity():
    """A logit of minus infinity is a token of probability 0; a row of nothing else has no gradient."""
    w = torch.zeros((200, 8), device="cuda").bfloat16()
    w[:, 0] = torch.linspace(-1, 1, 200).bfloat16()
    w[7, 1], w[150, 1] = float("-inf"), float("-inf")
    x = torch.zeros((3, 8), device="cuda").bfloat16()
    x[:, 0], x[:, 1] = torch.tensor([1.0, 2.0, 0.5]).cuda(), 1.0
    x[2, 1] = 0.5
    ids = torch.tensor([7, 3, 150], dtype=torch.int32, device="cuda")
    got = tt.head_logprobs(200, x, w, ids)
    z = x.double() @ torch.where(torch.isinf(w), torch.zeros_like(w), w).double().T
    z[:, [7, 150]] = -math.inf
    assert torch.allclose(got.lse.double(), torch.logsumexp(z, 1), atol=1e-5)
    assert got.logprob[0] == -math.inf and got.logprob[2] == -math.inf and bool(torch.isfinite(got.logprob[1]))
    w[:, 1] = float("-inf")
    got = tt.head_logprobs(200, x, w, ids)
    assert bool((got.lse == -math.inf).all()) and bool((got.logprob == -math.inf).all()) and not bool(got.stats[:, 1].any())
    dx, dw = tt.head_logprobs_backward(200, x, w, ids, got.stats, torch.ones(3, device="cuda"))
    assert not bool(dx.any()) and not bool(dw.any())


def test_ids_outside_the_vocabulary():
    x, w, ids, beta = uh.operands(6, 100, 16, "bf16")
    ids[1], ids[4] = -1, 100
    got = check_forward(100, x, w, ids, beta, "bf16")
    assert torch.isnan(got.logprob).tolist() == [False, True, False, False, True, False]


def test_outputs_in_the_callers_memory():
    """Rows further apart: what lies between them is left alone."""
    for name in ("bf16", "f16", "f32"):
        x, w, ids, beta = uh.operands(70, 200, 50, name)
        g, _ = weights(70)
        f = tt.HeadLogProbs(*(torch.full(k, 7.0, device="cuda") for k in ((70,), (70,), (70, 2))))
        got = check_forward(200, x, w, ids, beta, name, out=f)
        assert got is f
        wide = torch.full((75, 61), 7.0, device="cuda").to(x.dtype), torch.full((203, 53), 7.0, device="cuda").to(x.dtype)
        check_backward(200, x, w, ids, f.stats, g, None, beta, name, dhidden=wide[0][:, 3:], dweight=wide[1])
        for t, n, c0 in ((wide[0], 70, 3), (wide[1], 200, 0)):
            assert bool((t[n:] == 7.0).all()) and bool((t[:, :c0] == 7.0).all()) and bool((t[:, c0 + 50:] == 7.0).all())
    few = tt.head_logprobs(200, x, w, ids, out=tt.HeadLogProbs(None, torch.empty(70, device="cuda"), None))
    assert few.logprob is None and torch.equal(few.lse, tt.head_logprobs(200, x, w).lse)


def test_no_rows():
    w = torch.randn((30, 8), device="cuda").bfloat16()
    x = torch.empty((0, 8), device="cuda").bfloat16()
    ids, none = torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, device="cuda")
    got = tt.head_logprobs(30, x, w, ids)
    assert got.lse.numel() == 0
    dw = torch.full((33, 11), 7.0, device="cuda").bfloat16()
    dx, _ = tt.head_logprobs_backward(30, x, w, ids, torch.empty((0, 2), device="cuda"), none, dweight=dw)
    assert dx.shape == (0, 8) and not bool(dw[:30, :8].any()) and bool((dw[30:] == 7.0).all()) and bool((dw[:, 8:] == 7.0).all())


def test_one_workspace_for_batches_of_any_size():
    v, h = 3000, 96
    for name in ("bf16", "f32"):
        x, w, ids, beta = uh.operands(700, v, h, name)
        g, _ = weights(700)
        a, b = tt.head_logprobs_workspace(700, v, h, x.dtype), tt.head_logprobs_backward_workspace(700, v, h, x.dtype)
        for n in (700, 257, 256, 129, 64, 33, 16, 3, 1):
            a.fill_(255)
            b.fill_(255)  # no initialisation: NaN everywhere
            some = ids[:n].contiguous(), beta[:n].contiguous(), g[:n].contiguous()
            got = tt.head_logprobs(v, x[:n], w, some[0], inv_temperature=some[1], workspace=a)
            want = tt.head_logprobs(v, x[:n], w, some[0], inv_temperature=some[1])
            assert all(torch.equal(s, t) for s, t in zip(got, want)), n
            grads = [tt.head_logprobs_backward(v, x[:n], w, some[0], got.stats, some[2], inv_temperature=some[1], workspace=space) for space in (b, None)]
            assert all(torch.equal(s, t) for s, t in zip(*grads)), n
            assert all(bool(torch.isfinite(t.float()).all()) for t in grads[0])


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("n,v,h", [(1, 700, 64), (16, 20011, 64), (17, 3000, 128), (64, 700, 65), (65, 129, 64), (130, 1000, 64), (200, 257, 64),
                                   (257, 600, 96), (320, 513, 64), (500, 2000, 63), (513, 700, 64), (700, 300, 256)])
def test_nothing_behind_the_workspace_is_touched(n, v, h, name):
    """Workspaces of exactly the bytes that the calls ask for, in memory whose rest stays as it was."""
    x, w, ids, beta = uh.operands(n, v, h, name)
    g, q = weights(n)
    code = {"bf16": 0, "f32": 2}[name]
    used = [tt._spread_bytes(f, n, v, h, code) for f in ("tt_head_logprobs_workspace_size", "tt_head_logprobs_backward_workspace_used")]
    rooms = [torch.full((b + (1 << 20),), 93, dtype=torch.uint8, device="cuda") for b in used]
    out = tt.head_logprobs(v, x, w, ids, inv_temperature=beta, workspace=rooms[0][:used[0]])
    got = tt.head_logprobs_backward(v, x, w, ids, out.stats, g, grad_lse=q, inv_temperature=beta, workspace=rooms[1][:used[1]])
    for room, b in zip(rooms, used):
        assert bool((room[b:] == 93).all())
    want = tt.head_logprobs_backward(v, x, w, ids, out.stats, g, grad_lse=q, inv_temperature=beta)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("n,v,h,name", [(3, 5001, 64, "bf16"), (200, 2000, 128, "bf16"), (40, 900, 72, "f16"), (150, 700, 65, "f32")])
def test_replayed_in_a_graph_on_new_inputs(n, v, h, name):
    held = list(uh.operands(n, v, h, name))
    g, q = weights(n)

    def step():
        f = tt.head_logprobs(v, held[0], held[1], held[2], inv_temperature=held[3])
        return [*f, *tt.head_logprobs_backward(v, held[0], held[1], held[2], f.stats, g, grad_lse=q, inv_temperature=held[3])]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        results = step()
    for seed in range(1, 5):
        new = uh.operands(n, v, h, name, seed)
        new[2][: n // 3] = -1
        for old, t in zip(held, new):
            old.copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(results, step()):
            assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b)), seed


def test_on_another_stream():
    x, w, ids, beta = uh.operands(90, 3000, 64, "bf16")
    g, _ = weights(90)
    want = tt.head_logprobs(3000, x, w, ids, inv_temperature=beta)
    grads = tt.head_logprobs_backward(3000, x, w, ids, want.stats, g, inv_temperature=beta)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = tt.head_logprobs(3000, x, w, ids, inv_temperature=beta, stream=side)
    also = tt.head_logprobs_backward(3000, x, w, ids, got.stats, g, inv_temperature=beta, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip([*want, *grads], [*got, *also]))


def test_a_training_step():
    """hidden and weights from earlier layers, masked prompts, label smoothing's place taken by a penalty on the log-sum-exp."""
    n, v, h = 96, 1500, 64
    base, w0, ids, _ = uh.operands(n, v, h, "f32")
    ids[:20] = -1
    layer = (torch.randn((h, h), generator=torch.Generator().manual_seed(1)) / 8).cuda().requires_grad_()
    head = w0.clone().requires_grad_()
    kept = (ids >= 0).float()
    g, q = -kept / kept.sum(), 1e-2 * kept / kept.sum()
    hidden = base @ layer
    f = tt.head_logprobs(v, hidden.detach(), head.detach(), ids)
    dx, dw = tt.head_logprobs_backward(v, hidden.detach(), head.detach(), ids, f.stats, g, grad_lse=q)
    hidden.backward(dx)
    head.grad = dw
    got = [layer.grad.double(), head.grad.double()]
    layer64, head64 = layer.detach().double().requires_grad_(), head.detach().double().requires_grad_()
    z = base.double() @ layer64 @ head64.T
    lse = torch.logsumexp(z, 1)
    lp = z.gather(1, ids.long().clamp_min(0)[:, None])[:, 0] - lse
    ((g * lp) + (q * lse)).sum().backward()
    for a, b in zip(got, (layer64.grad, head64.grad)):
        assert float((a - b).norm() / b.norm()) < 1e-5


def test_written_tensors_are_reported_to_autograd():
    x, w, ids, beta = uh.operands(6, 100, 16, "f32")
    out = tt.head_logprobs(100, x, w, ids)
    g = torch.ones(6, device="cuda")
    grads = tt.head_logprobs_backward(100, x, w, ids, out.stats, g)
    for t, again in ((out.lse, lambda: tt.head_logprobs(100, x, w, ids, out=out)),
                     (grads[1], lambda: tt.head_logprobs_backward(100, x, w, ids, out.stats, g, dhidden=grads[0], dweight=grads[1]))):
        scale = torch.ones(1, device="cuda", requires_grad=True)
        y = (t * scale).sum()
        again()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
