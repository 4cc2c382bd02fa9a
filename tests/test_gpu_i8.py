"""tt_quantize_i8 and tt_matmul_i8 against their definitions, and the head in 8 bits from hidden states to the verification."""
import math

import numpy as np
import pytest
import torch

import paper_2510_15545_amd as tt
import util_head as uh

pytestmark = pytest.mark.gpu

NAN, U = float("nan"), 2.0 ** -24


def definition(x):
    """(q, scale) in numpy: fp32 quotients, each rounded once (torch multiplies by a scalar divisor's reciprocal)."""
    f = x.float().cpu().numpy()
    with np.errstate(all="ignore"):
        scale = np.abs(f).max(1) / np.float32(127.0)
        bad = ~np.isfinite(f).all(1)
        none = bad | (scale == 0)
        q = np.clip(np.rint(f / np.where(none, np.float32(1.0), scale)[:, None]), -127, 127)
    q[none] = 0
    return torch.from_numpy(q.astype(np.int8)).cuda(), torch.from_numpy(np.where(bad, np.float32(NAN), scale).astype(np.float32)).cuda()


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,k", [(1, 1), (1, 2048), (3, 7), (5, 64), (70, 1000), (9, 4097), (2, 16384), (1, 131071), (3, 33333), (700, 256)])
def test_quantize(n, k, name):
    gen = torch.Generator().manual_seed(n * k)
    x = (torch.randn((n, k), generator=gen) * torch.logspace(-3, 2, n)[:, None]).to(uh.TYPES[name]).cuda()
    for pad, shift in ((0, 0), (8, 0), (3, 1)):
        print(f"[case] {n}x{k} {name} pad {pad} shift {shift}", flush=True)
        q, scale = tt.quantize_i8(uh.placed(x, pad, shift))
        want = definition(x)
        assert torch.equal(q, want[0]) and torch.equal(scale, want[1])


def test_quantize_rows_of_every_kind():
    x = torch.randn((9, 300), generator=torch.Generator().manual_seed(1)).cuda()
    x[0] = 0.0
    x[1, 7] = NAN
    x[2, 299] = float("inf")
    x[3, 0] = -float("inf")
    x[4] = 1e-45
    x[5] *= 3e38 / float(x[5].abs().max())
    x[6] = -3.0
    x[7] *= 1e-38
    out = torch.full((12, 310), 5, dtype=torch.int8, device="cuda"), torch.full((9,), 5.0, device="cuda")
    q, scale = tt.quantize_i8(x, out=(out[0][:9, 4:304], out[1]))
    want = definition(x)
    assert torch.equal(torch.isnan(scale), torch.isnan(want[1])) and torch.equal(torch.nan_to_num(scale), torch.nan_to_num(want[1]))
    assert torch.equal(q, want[0])
    assert bool((out[0][9:] == 5).all()) and bool((out[0][:, :4] == 5).all()) and bool((out[0][:, 304:] == 5).all())
    q, scale = tt.quantize_i8(torch.empty((0, 300), device="cuda"))
    assert q.shape == (0, 300) and scale.shape == (0,)


def ints(n, k, seed, low=-128):
    gen = torch.Generator().manual_seed(seed)
    return torch.randint(low, 128, (n, k), generator=gen, dtype=torch.int8).cuda()


def scales(n, seed, size):
    return ((0.5 + torch.rand(n, generator=torch.Generator().manual_seed(seed))) * size).cuda()


def check_matmul(x, xs, w, ws, bias, name, beta=None, lse=False, **kw):
    dtype = uh.TYPES[name]
    out, got = tt.matmul_i8(x, xs, w, ws, bias=bias, dtype=dtype, lse=lse, inv_temperature=beta, **kw)
    total = x.double() @ w.double().T  # exact
    y = total * xs.double()[:, None] * ws.double()
    off = 4 * U * y.abs()  # the conversion and two products
    if bias is not None:
        y = y + bias.double()
        off = off + U * y.abs()
    want = out.double()
    # rounded once: no further from the value than half a step of the type, measured at the result
    half = uh.HALF_STEP[name] * y.abs() + off * (1 + uh.HALF_STEP[name])
    if name == "f16":
        half = half + 2.0 ** -25
    assert bool(((want - y).abs() <= half).all()), float(((want - y).abs() - half).max())
    if lse is not False:
        b = torch.ones(len(x), dtype=torch.float64, device="cuda") if beta is None else beta.double()
        z = want * b[:, None]
        total = torch.logsumexp(z, 1)
        m = z.amax(1)
        off = U * (300 + 12 * math.log(z.shape[1] + 1) + 8) + 2 * U * (total.abs() + m.abs() + (total - m).abs())
        assert bool(((got.double() - total).abs() <= off).all()), float(((got.double() - total).abs() - off).max())
    else:
        assert got is None
    return out, got


SIZES = [(1, 1, 1), (1, 640, 256), (2, 3, 5), (3, 129, 65), (16, 513, 64), (17, 300, 130), (33, 77, 128), (64, 1025, 200), (65, 257, 1000),
         (130, 384, 64), (257, 130, 96), (300, 500, 4096), (5, 20011, 48), (1, 5000, 4096), (129, 128, 16), (40, 33, 15),
         (12, 333, 2048), (16, 100, 5000), (7, 50, 9216), (3, 40, 70000), (520, 700, 256), (200, 1000, 384)]


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,m,k", SIZES)
def test_matmul_sizes_and_layouts(n, m, k, name):
    x, w = ints(n, k, 1), ints(m, k, 2)
    xs, ws = scales(n, 3, 0.05), scales(m, 4, 2.0 / math.sqrt(k) / 127)
    bias, beta = torch.randn(m, generator=torch.Generator().manual_seed(5)).cuda(), scales(n, 6, 1.0)
    for pad, shift in ((0, 0), (16, 0), (3, 1)):
        print(f"[case] {n}x{m}x{k} {name} pad {pad} shift {shift}", flush=True)
        xp, wp = uh.placed(x, pad, shift, 77.0), uh.placed(w, pad, shift, 77.0)
        check_matmul(xp, xs, wp, ws, None, name, beta, lse=True)
        wide = torch.full((n + 2, m + pad), 7.0, device="cuda").to(uh.TYPES[name])
        check_matmul(xp, xs, wp, ws, bias, name, out=wide[:, :m][:n] if pad else None)
        if pad:
            assert bool((wide[n:] == 7.0).all()) and bool((wide[:, m:] == 7.0).all())


def test_integers_are_exact():
    """Sums at the ends of 32 bits, and beyond fp32's whole numbers: the result is the exact sum, rounded once."""
    k = 131071
    x = torch.full((3, k), -128, dtype=torch.int8, device="cuda")
    x[1] = 127
    x[2] = ints(1, k, 9)[0]
    w = torch.full((20, k), -128, dtype=torch.int8, device="cuda")
    w[5:] = ints(15, k, 10)
    one = torch.ones(20, device="cuda")
    out, _ = tt.matmul_i8(x, one[:3].contiguous(), w, one, dtype=torch.float32)
    want = torch.from_numpy((x.cpu().numpy().astype(np.int64) @ w.cpu().numpy().astype(np.int64).T)).cuda()
    assert int(want.max()) > 2 ** 30
    assert torch.equal(out, want.float())


def test_log_sum_exp_of_rows_of_every_kind():
    x, w = ints(140, 64, 1), ints(300, 64, 2)
    xs, ws = scales(140, 3, 0.01), scales(300, 4, 0.01)
    beta = scales(140, 6, 1.0)
    _, want = tt.matmul_i8(x, xs, w, ws, lse=True, inv_temperature=beta)
    xs[3], xs[100], beta[50], beta[60], beta[70], beta[139] = NAN, float("inf"), 0.0, NAN, -2.0, 2.0 ** 101
    out, got = tt.matmul_i8(x, xs, w, ws, lse=True, inv_temperature=beta)
    bad = [3, 50, 60, 70, 100, 139]
    good = torch.ones(140, dtype=torch.bool)
    good[bad] = False
    assert bool(torch.isnan(got[bad]).all()) and torch.equal(got[good], want[good]) and bool(torch.isnan(out[3]).all())
    # all logits far below zero
    low = torch.full((300,), -5000.0, device="cuda")
    for n in (3, 20, 40, 100, 140):
        check_matmul(x[:n], scales(n, 3, 0.01), w, ws, low, "f32", lse=True)
    # equal logits: ln of their number
    zero = torch.zeros_like(x)
    _, got = tt.matmul_i8(zero, torch.ones(140, device="cuda"), w, ws, lse=True)
    assert bool(((got - math.log(300)).abs() < 1e-5).all())
    # a bias of minus infinity masks a token, and all of them the row
    bias = torch.zeros(300, device="cuda")
    bias[10:] = -float("inf")
    _, got = tt.matmul_i8(zero, torch.ones(140, device="cuda"), w, ws, bias=bias, lse=True)
    assert bool(((got - math.log(10)).abs() < 1e-5).all())
    bias[:] = -float("inf")
    out, got = tt.matmul_i8(zero, torch.ones(140, device="cuda"), w, ws, bias=bias, lse=True)
    assert bool((got == -float("inf")).all()) and bool((out == -float("inf")).all())


def test_scales_of_the_same_rows_given_twice():
    """One memory for both operands."""
    x = ints(70, 96, 1)
    s = scales(70, 2, 0.02)
    check_matmul(x, s, x, s, None, "f32", lse=True)


def test_no_rows_and_the_callers_memory():
    w, ws = ints(50, 32, 1), scales(50, 2, 0.1)
    out, lse = tt.matmul_i8(torch.empty((0, 32), dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda"), w, ws, lse=True)
    assert out.shape == (0, 50) and lse.shape == (0,)
    x, xs = ints(600, 32, 3), scales(600, 4, 0.1)
    space = tt.matmul_i8_workspace(600, 50, 32, lse=True)
    for n in (600, 257, 128, 33, 16, 1):
        space.fill_(255)
        mine = torch.empty((n, 50), device="cuda").half(), torch.empty(n, device="cuda")
        got = tt.matmul_i8(x[:n], xs[:n].contiguous(), w, ws, out=mine[0], lse=mine[1], workspace=space)
        want = tt.matmul_i8(x[:n], xs[:n].contiguous(), w, ws, dtype=torch.float16, lse=True)
        assert got[0] is mine[0] and got[1] is mine[1] and all(torch.equal(a, b) for a, b in zip(got, want)), n


@pytest.mark.parametrize("n,m,k", [(1, 700, 64), (16, 20011, 64), (17, 3000, 128), (64, 700, 65), (100, 129, 128), (200, 257, 128), (300, 600, 200),
                                   (320, 513, 128)])
def test_nothing_behind_the_workspace_is_touched(n, m, k):
    x, w = ints(n, k, 1), ints(m, k, 2)
    xs, ws = scales(n, 3, 0.05), scales(m, 4, 0.01)
    b = tt.matmul_i8_workspace(n, m, k, lse=True).numel()
    room = torch.full((b + (1 << 20),), 93, dtype=torch.uint8, device="cuda")
    got = tt.matmul_i8(x, xs, w, ws, lse=True, workspace=room[:b])
    assert bool((room[b:] == 93).all())
    assert all(torch.equal(s, t) for s, t in zip(got, tt.matmul_i8(x, xs, w, ws, lse=True)))


def test_on_another_stream_and_in_a_graph():
    x, xs, w, ws = ints(100, 128, 1), scales(100, 2, 0.05), ints(900, 128, 3), scales(900, 4, 0.01)
    want = tt.matmul_i8(x, xs, w, ws, lse=True)
    hidden = torch.randn((100, 128), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = tt.matmul_i8(x, xs, w, ws, lse=True, stream=side)
    q = tt.quantize_i8(hidden, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got)) and all(torch.equal(a, b) for a, b in zip(q, tt.quantize_i8(hidden)))

    def step():
        return tt.matmul_i8(*tt.quantize_i8(hidden), w, ws, lse=True)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        results = step()
    for seed in range(2, 6):
        hidden.copy_(torch.randn((100, 128), generator=torch.Generator().manual_seed(seed)) * seed)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(results, step())), seed


@pytest.mark.parametrize("with_workspace", [False, True])
def test_the_head_in_8_bits_before_the_verification(with_workspace, orc):
    """Hidden states quantised, multiplied with quantised weights, their logits and log-sum-exp verified: the oracle's results on the
    same logits and log-sum-exp."""
    n_streams, m, v, h = 12, 4, 3001, 128
    rows = n_streams * (m + 1)
    x, w, ids, _ = uh.operands(rows, v, h, "bf16", lean=10.0)
    wq = tt.quantize_i8(w)
    inv_t = scales(n_streams, 1, 1.2)
    beta = inv_t.repeat_interleave(m + 1)
    logits, lse = tt.matmul_i8(*tt.quantize_i8(x), *wq, lse=True, inv_temperature=beta)
    full = (x.double() @ w.double().T)
    assert float((logits.double() - full).abs().max()) < 0.02 * float(full.abs().max()) + 0.1
    rng = np.random.default_rng(3)
    off = torch.arange(0, n_streams * m + 1, m, dtype=torch.int32, device="cuda")
    target = ids.view(n_streams, m + 1)[:, :m].reshape(-1).contiguous()
    q = torch.from_numpy(rng.random(n_streams * m).astype(np.float32) * 0.5).cuda()
    ua, us = (torch.from_numpy(rng.random(k).astype(np.float32)).cuda() for k in (n_streams * m, n_streams))
    space = tt.verify_logits_workspace(n_streams, v, m, lse=True) if with_workspace else torch.empty(0, dtype=torch.uint8, device="cuda")
    got = tt.verify_logits(v, target, off, q, logits, inv_t, ua, us, m, lse=lse, workspace=space)
    torch.cuda.synchronize()
    host = lambda t: t.cpu().numpy()  # noqa: E731
    want = orc.verify_logits(v, host(target), host(off), host(q), host(logits.view(torch.int16)).view(np.uint16), host(inv_t), host(ua), host(us), m,
                             lse=host(lse))
    assert np.array_equal(host(got[0]), want[0]) and np.array_equal(host(got[1]), want[1])
