"""The output head and the 8-bit product at sizes of every tile shape, over several pieces of a vocabulary and several launches of rows,
against the definitions in 64 bits."""
import math

import pytest
import torch

import paper_2510_15545_amd as tt
import util_head as uh
import util_head_sizes as sizes
from test_gpu_head import check_forward, close
from test_gpu_i8 import check_matmul, ints, scales

pytestmark = pytest.mark.gpu

LAYOUTS = [(0, 0), (8, 0)]  # of rows further apart: 16-byte aligned ones both


def edges(ids, v):
    """Tokens at the vocabulary's ends among the rows' own, the last two rows' beside each other."""
    ids = ids.clone()
    ids[0], ids[1], ids[-1] = v - 1, 0, v - 2
    return ids


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,v,h", sizes.FORWARD)
def test_log_probabilities(n, v, h, name):
    x, w, ids, beta = uh.operands(n, v, h, name)
    ids = edges(ids, v)
    for pad, shift in LAYOUTS:
        print(f"[case] {n}x{v}x{h} {name} pad {pad}", flush=True)
        check_forward(v, uh.placed(x, pad, shift), uh.placed(w, pad, shift), ids, beta, name)
    ids[2], ids[n // 2] = -1, v
    got = check_forward(v, x, w, ids, None, name)
    assert int(torch.isnan(got.logprob).sum()) == 2


def check_gradient(n, v, h, name, seed=0, pad=0):
    x, w, ids, beta = uh.operands(n, v, h, name, seed)
    ids = edges(ids, v)
    gen = torch.Generator().manual_seed(n + seed)
    g, q = (torch.rand(n, generator=gen) + 0.5).cuda(), torch.randn(n, generator=gen).cuda()
    for out, q2 in ((0.0, None), (0.3, None), (0.0, q)):
        print(f"[case] {n}x{v}x{h} {name} pad {pad}, {out} without a weight, log-sum-exp {q2 is not None}", flush=True)
        some = ids.clone()
        some[torch.randperm(n, generator=gen)[:int(out * n)].cuda()] = -1
        xs, ws = uh.placed(x, pad), uh.placed(w, pad)
        stats = tt.head_logprobs(v, xs, ws, some, inv_temperature=beta).stats
        got = tt.head_logprobs_backward(v, xs, ws, some, stats, g, grad_lse=q2, inv_temperature=beta)
        want = uh.backward(x, w, some, stats, g, q2, beta, name)
        for a, b, off, what in zip(got, want[:2], want[2:], ("dhidden", "dweight")):
            close(a, b, off, what)
            if name != "f32":  # and one rounding of the result as a whole: see test_gradients_are_rounded_once
                once = float((b.to(a.dtype).double() - b).norm() / b.norm())
                assert float((a.double() - b).norm() / b.norm()) <= once + uh.HALF_STEP[name] / 16, what


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,v,h", sizes.GRADIENT)
def test_gradients(n, v, h, name):
    check_gradient(n, v, h, name)
    check_gradient(n, v, h, name, seed=1, pad=8)


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,v,h", sizes.PIECES)
def test_gradients_over_several_pieces(n, v, h, name):
    check_gradient(n, v, h, name)


@pytest.mark.parametrize("name", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("n,m,k", [(n, v, 128 if h == 64 else 256) for n, v, h in sizes.FORWARD])
def test_8_bit_product(n, m, k, name):
    x, w = ints(n, k, 1), ints(m, k, 2)
    xs, ws = scales(n, 3, 0.05), scales(m, 4, 2.0 / math.sqrt(k) / 127)
    bias, beta = torch.randn(m, generator=torch.Generator().manual_seed(5)).cuda(), scales(n, 6, 1.0)
    for pad in (0, 16):
        print(f"[case] {n}x{m}x{k} {name} pad {pad}", flush=True)
        xp, wp = uh.placed(x, pad, 0, 77.0), uh.placed(w, pad, 0, 77.0)
        check_matmul(xp, xs, wp, ws, bias, name, beta, lse=True)
        wide = torch.full((n + 2, m + 5), 7.0, device="cuda").to(uh.TYPES[name])
        check_matmul(xp, xs, wp, ws, None, name, out=wide[:n, :m])
        assert bool((wide[n:] == 7.0).all()) and bool((wide[:, m:] == 7.0).all())


ROWS = (1 << 14) + 70  # more than a launch takes


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("h", [64, 60])
def test_log_probabilities_and_gradients_of_many_rows(h, name):
    x, w, ids, beta = uh.operands(ROWS, 301, h, name)
    ids = edges(ids, 301)
    got = check_forward(301, x, w, ids, beta, name)
    g = (torch.rand(ROWS, generator=torch.Generator().manual_seed(1)) + 0.5).cuda()
    g[5::3] = 0.0
    dx, dw = tt.head_logprobs_backward(301, x, w, ids, got.stats, g, inv_temperature=beta)
    want = uh.backward(x, w, ids, got.stats, g, None, beta, name)
    close(dx, want[0], want[2], "dhidden")
    close(dw, want[1], want[3], "dweight")
    assert not bool(dx[5::3].any())


@pytest.mark.parametrize("k", [128, 120])
def test_8_bit_product_of_many_rows(k):
    x, w = ints(ROWS, k, 1), ints(301, k, 2)
    xs, ws = scales(ROWS, 3, 0.05), scales(301, 4, 2.0 / math.sqrt(k) / 127)
    bias = torch.randn(301, generator=torch.Generator().manual_seed(5)).cuda()
    check_matmul(x, xs, w, ws, bias, "bf16", scales(ROWS, 6, 1.0), lse=True)
