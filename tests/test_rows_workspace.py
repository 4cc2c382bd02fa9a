"""Workspaces of the calls on rows of logits: one taken for the largest batch serves the smaller ones."""
import ctypes

import pytest

import paper_2510_15545_amd as tt

BF16, F32 = 0, 2
ROWS = [1, 2, 3, 7, 40, 60, 64, 90, 95, 96, 97, 128, 150, 191, 192, 193, 300, 700, 1023, 1024, 1025, 3000, 5001]


def query(name, *sizes):
    n = ctypes.c_size_t(0)
    assert getattr(tt.lib(), name)(*sizes, ctypes.byref(n)) == tt.TT_OK
    return n.value


def check(op, rows, *sizes):
    """The size never falls with the rows, and no number of rows up to them uses more."""
    size = [query(f"tt_{op}_workspace_size", n, *sizes) for n in rows]
    assert size == sorted(size), (op, sizes, size)
    used = [query(f"tt_{op}_workspace_used", n, *sizes) for n in rows]
    for i, most in enumerate(size):
        assert max(used[:i + 1]) <= most, (op, sizes, rows[i])


@pytest.mark.parametrize("v,dtype", [(640, BF16), (65536, BF16), (65537, BF16), (70001, BF16), (128256, BF16), (151936, F32), (300007, BF16),
                                     (600000, F32), (1 << 23, BF16)])
def test_a_workspace_for_more_rows_serves_fewer(v, dtype):
    for n_top in (0, 20, 128):
        check("logprobs", ROWS, v, dtype, n_top)
    for grad in (0, 1):
        check("distill", ROWS, v, dtype, 64, grad)


def test_every_number_of_rows():
    check("logprobs", list(range(0, 260)), 128256, BF16, 20)
    check("distill", list(range(0, 260)), 151936, BF16, 64, 1)
    check("distill", list(range(0, 2100)), 300000, BF16, 64, 1)
    check("distill", list(range(0, 2100)), 300000, BF16, 64, 0)
    # groups of rows: several of 18 rows, and 2^18 / 2 rows of two parts
    check("distill", list(range(0, 200)), 1 << 20, F32, 7, 1)
    check("distill", [100000, 131071, 131072, 131073, 200000, 262144, 262145, 2 ** 31 - 1], (1 << 18) + 1, BF16, 7, 0)


def test_fewer_tokens_use_less():
    for n in (1, 48, 95):
        for op, more in (("logprobs", ()), ("distill", (1,))):
            sizes = [query(f"tt_{op}_workspace_size", n, 151936, BF16, k, *more) for k in (1, 2, 20, 64, 128)]
            assert sizes == sorted(sizes)


def test_refusals():
    n = ctypes.c_size_t(0)
    L = tt.lib()
    for bad in ((-1, 100, 0, 3), (2, 0, 0, 3), (2, 100, 5, 3), (2, 100, 0, -1)):
        assert L.tt_logprobs_workspace_used(*bad, ctypes.byref(n)) == tt.TT_EINVAL
        assert L.tt_distill_workspace_used(*bad, 1, ctypes.byref(n)) == tt.TT_EINVAL
    assert L.tt_distill_workspace_used(2, 100, 0, 0, 1, ctypes.byref(n)) == tt.TT_EINVAL
    for bad in ((2, (1 << 23) + 1, 0, 3), (2, 100, 0, 129)):
        assert L.tt_logprobs_workspace_used(*bad, ctypes.byref(n)) == tt.TT_EUNSUPPORTED
        assert L.tt_distill_workspace_used(*bad, 0, ctypes.byref(n)) == tt.TT_EUNSUPPORTED
    assert L.tt_logprobs_workspace_used(2, 100, 0, 3, None) == tt.TT_EINVAL
    assert L.tt_distill_workspace_used(2, 100, 0, 3, 1, None) == tt.TT_EINVAL


@pytest.mark.gpu
@pytest.mark.parametrize("v", [128256, 300007])
def test_one_workspace_for_batches_of_any_size(v):
    import torch

    most, k = 210, 20
    g = torch.Generator(device="cuda").manual_seed(v)
    rows = torch.randn((most, v), device="cuda", generator=g).mul_(3).bfloat16()
    ids = torch.randint(0, v, (most, k), device="cuda", generator=g, dtype=torch.int32)
    lp = torch.randn((most, k), device="cuda", generator=g) - 5
    w = torch.rand(most, device="cuda", generator=g)
    space = tt.logprobs_workspace(most, v, rows.dtype, k)
    room = tt.distill_workspace(most, v, rows.dtype, k, grad=True)
    for n in (210, 192, 191, 100, 96, 95, 90, 64, 60, 9, 1):
        print(f"[case] {n} of {most} rows of {v}", flush=True)
        few = rows[:n], ids[:n].contiguous(), lp[:n].contiguous(), w[:n].contiguous()
        got = tt.logprobs(v, few[0], few[1][:, 0].contiguous(), n_top=k, entropy=True, workspace=space)
        want = tt.logprobs(v, few[0], few[1][:, 0].contiguous(), n_top=k, entropy=True)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), n
        got = tt.distill(v, *few[:3], tail=True, grad_loss=few[3], workspace=room)
        want = tt.distill(v, *few[:3], tail=True, grad_loss=few[3])
        assert all(torch.equal(a, b) for a, b in zip(got, want)), n
