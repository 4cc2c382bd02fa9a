"""Rows of logits that several workgroups share, few long ones: masks, NaN, lists and temperatures of every kind where
the parts meet, parts without a token, more parts than a workgroup has threads, selections that do not fit."""
import numpy as np
import pytest
import torch

import util_rows as ur
from test_gpu_distill import check, lists
from test_gpu_logprobs import check_gradient, check_logprobs

pytestmark = pytest.mark.gpu

TYPES = ["bf16", "f16", "f32"]
WIDE = {"bf16": 70001, "f16": 70001, "f32": 40001}  # 9 or 10 parts of 16 KB, the last of a row's end
PART = {"bf16": 8192, "f16": 8192, "f32": 4096}
LOWEST = {"bf16": -3.3895313892515355e38, "f16": -65504.0, "f32": -3.4028234663852886e38}


def split(op, n, v, dtype, k):
    """That these rows are split."""
    import paper_2510_15545_amd as tt

    sizes = (n, v, ("bf16", "f16", "f32").index(dtype), k) + ((1,) if op == "distill" else ())
    return tt._spread_bytes(f"tt_{op}_workspace_used", *sizes) > 0


def masked_rows(rng, dtype):
    """Rows held to tokens in one part, in some, in the first or last of each, at the parts' borders, in runs."""
    v, part = WIDE[dtype], PART[dtype]
    kept = [np.arange(0), np.array([v - 1]), np.array([part]), np.array([0, part - 1, part, 2 * part - 1, v - 1]),
            part + np.arange(7), 3 * part + np.arange(300), part - 100 + np.arange(256), 2 * part + np.arange(part),
            np.arange(0, v, part), v - 1 - np.arange(400), rng.permutation(v)[:20], rng.permutation(v)[:129], rng.permutation(v)[:6000]]
    rows = []
    for at in kept:
        for mask in (-np.inf, np.nan, max(-1e9, LOWEST[dtype]), LOWEST[dtype]):
            x = np.full(v, mask, np.float32)
            x[at] = rng.standard_normal(len(at)) * 3
            rows.append(x)
    return np.array(rows)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n_top", [0, 1, 20, 128])
def test_masks(dtype, n_top):
    rng = np.random.default_rng(31)
    x = masked_rows(rng, dtype)
    n, v = x.shape
    assert split("logprobs", n, v, dtype, n_top)
    ids = rng.integers(0, v, n)
    ids[::2] = [np.nanargmax(np.where(np.isnan(r), -np.inf, r)) for r in x[::2]]
    got = check_logprobs(x, ur.placed(x, dtype, pad=3, shift=1), ids, (0.5 + rng.random(n)).astype(np.float32), n_top)
    assert ur.host(got.lse)[0] == -np.inf and ur.host(got.entropy)[0] == 0.0


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_without_a_distribution(dtype):
    rng = np.random.default_rng(32)
    v = WIDE[dtype]
    x = ur.model_rows(rng, 12, v)
    x[1, 17], x[2, v - 1] = np.inf, np.inf
    x[3] = -np.inf
    x[3, PART[dtype]] = np.inf
    x[4] = np.nan
    beta = np.array([1.0, 1.0, 1.0, 1.0, 1.0, 0.0, -1.0, np.nan, np.inf, 2.0 ** 101, 2.0 ** 100, 2.0], np.float32)
    ids = np.array([-1, 17, 3, 4, 5, 6, 7, 8, 9, 10, x[10].argmax(), v])
    x[10, [5, v - 9, PART[dtype]]] = x[10].max()  # equal largest logits in three parts at the steepest temperature
    for n_top in (0, 5, 128):
        assert split("logprobs", len(x), v, dtype, n_top)
        check_logprobs(x, ur.placed(x, dtype), ids, beta, n_top)


@pytest.mark.parametrize("n_top", [1, 20, 128])
@pytest.mark.parametrize("dtype", TYPES)
def test_equal_logits_go_to_the_lower_token(dtype, n_top):
    """More equal keys than the joining kernel orders, plateaus over the parts' borders, rows that rise or fall."""
    rng = np.random.default_rng(33)
    v, part = WIDE[dtype], PART[dtype]
    at = np.arange(v)
    x = np.zeros((9, v), np.float32)
    x[1] = rng.integers(0, 2, v)
    x[2] = np.minimum(rng.standard_normal(v) * 3, 4.0)
    x[3] = np.where((at > part - 50) & (at < part + 50), 5.0, rng.standard_normal(v))
    x[4] = at // 512
    x[5] = -(at // 512)
    x[6] = np.where(at % 2048 < 8, 6.0, 0.0) + (at % 2048 == 5)
    x[7] = np.where(at >= v - 300, 2.0, 0.0)
    x[8] = at % part // 64  # every part the same
    x = np.round(x * 4) / 4
    assert split("logprobs", len(x), v, dtype, n_top)
    check_logprobs(x, ur.placed(x, dtype, pad=1), rng.integers(0, v, len(x)), None, n_top)


@pytest.mark.parametrize("v,dtype,n_top", [(147856, "bf16", 20), (147856, "bf16", 32), (131584, "f16", 20), (73744, "f32", 12), (65736, "bf16", 8)])
def test_a_last_part_with_few_tokens(v, dtype, n_top):
    """Fewer groups of threads than alternatives have a token of the last part, more tokens than it may hand over."""
    rng = np.random.default_rng(v)
    x = ur.model_rows(rng, 2, v)
    assert split("logprobs", 2, v, dtype, n_top)
    check_logprobs(x, ur.placed(x, dtype), rng.integers(0, v, 2), None, n_top)


@pytest.mark.parametrize("v,dtype,n_top", [((1 << 22) + 3, "bf16", 128), ((1 << 22) + 3, "f32", 20), (1 << 23, "bf16", 0), (1 << 23, "f32", 128)])
def test_more_parts_than_threads(v, dtype, n_top):
    print(f"[case] 1x{v} {dtype} top {n_top}", flush=True)
    rng = np.random.default_rng([v, n_top])
    x = ur.model_rows(rng, 1, v)
    x[0, -3:] = 12.5
    assert split("logprobs", 1, v, dtype, n_top)
    rows = ur.placed(x, dtype, shift=1)
    check_logprobs(x, rows, np.array([v - 1]), np.full(1, 0.9, np.float32), n_top)
    check_gradient(x, rows, np.array([v - 1]), None, np.ones(1, np.float32), np.ones(1, np.float32), dtype)


@pytest.mark.parametrize("v,dtype", [((1 << 22) + 3, "bf16"), (1 << 23, "f32")])
def test_distillation_of_more_parts_than_threads(v, dtype):
    print(f"[case] distill 1x{v} {dtype}", flush=True)
    rng = np.random.default_rng(v)
    k = 128
    x = ur.model_rows(rng, 1, v)
    ids, lp = lists(rng, 1, v, k)
    ids[0, 5], ids[0, 6], ids[0, 9] = v - 1, 0, v - 1
    x[0, ids[0]] = 14.0 + lp[0]
    assert split("distill", 1, v, dtype, k)
    check(ur.placed(x, dtype, shift=1), ids, lp, None, True, np.ones(1, np.float32), dtype)
    check(ur.placed(x, dtype), ids, lp, None, True, None, dtype)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k", [24, 100])
def test_lists_of_every_kind(dtype, tail, k):
    rng = np.random.default_rng(34)
    n, v = 18, WIDE[dtype]
    x = ur.model_rows(rng, n, v)
    ids, lp = lists(rng, n, v, k)
    ids[1, :] = 5  # one token only
    ids[2, ::2] = ids[2, 1::2]  # each twice
    ids[3, :] = -1  # nothing
    ids[4, :] = v
    ids[5, 3:] = -1
    lp[6, :] = -np.inf
    lp[7, ::3] = np.nan
    lp[8, 4:] = -np.inf
    lp[9, 5] = np.inf
    lp[10] += 3.0  # masses that sum to more than 1
    lp[11] -= 90.0  # hardly any mass
    lp[12, 1:] = -200.0
    x[13, ids[13, 3]] = -np.inf  # a listed token that the student excludes: an infinite loss
    ids[14, 7], ids[15, 7] = 2 ** 31 - 1, -2 ** 31
    ids[16, -1] = ids[16, 0]  # the first and the last entry
    ids[17, :] = np.arange(k) % 3 + PART[dtype] - 1  # three tokens around a border
    weight = rng.standard_normal(n).astype(np.float32)
    assert split("distill", n, v, dtype, k)
    loss, grad = check(ur.placed(x, dtype, pad=1), ids, lp, None, tail, weight, dtype)
    for i in (3, 4, 6):
        assert ur.host(loss)[i] == 0.0 and not ur.host(grad)[i].any()
    assert np.isnan(ur.host(loss)[9]) and ur.host(loss)[13] == np.inf


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_distillation_of_masked_and_unsound_rows(dtype, tail):
    rng = np.random.default_rng(35)
    lowest, part = LOWEST[dtype], PART[dtype]
    n, v, k = 20, WIDE[dtype], 12
    x = ur.model_rows(rng, n, v)
    ids, lp = lists(rng, n, v, k)
    x[1] = -np.inf
    x[2] = np.nan
    x[3] = lowest
    x[4], x[4, ids[4]] = -np.inf, rng.standard_normal(k)  # only listed tokens left
    x[5], x[5, ids[5]] = lowest, rng.standard_normal(k)
    x[6, ids[6]], x[6, 9] = 1.0, np.inf
    x[7, ids[7, 2]] = np.inf
    x[12, ids[12]] = 300.0  # hardly any mass outside the list
    x[13, ids[13]] = -300.0  # hardly any inside
    x[14] = max(lowest, -1e9)
    x[15, ids[15]] = np.nan
    x[16, part:2 * part] = -np.inf  # parts without a token
    x[17, :part] = np.nan
    x[18, part:] = -np.inf
    x[19, v - v % part:] = -np.inf
    beta = np.ones(n, np.float32)
    beta[8:12] = 0.0, -2.0, np.nan, np.inf
    weight = rng.standard_normal(n).astype(np.float32)
    assert split("distill", n, v, dtype, k)
    rows = ur.placed(x, dtype, pad=2)
    loss, grad = check(rows, ids, lp, beta, tail, weight, dtype)
    for i in (1, 2):
        assert ur.host(loss)[i] == 0.0 and not ur.host(grad)[i].any()
    weight[6:12] = 0.0  # padded rows: weight 0 gives zeros whatever the row holds
    _, grad = check(rows, ids, lp, beta, tail, weight, dtype)
    assert not ur.host(grad)[6:12].any()
    check(rows, ids, lp, beta, tail, weight, dtype, out=rows)  # in place


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
def test_lists_of_another_vocabulary(dtype, tail):
    rng = np.random.default_rng(36)
    n, v, other, k = 9, WIDE[dtype], 50021, 50
    x = ur.model_rows(rng, n, v)
    ids, lp = lists(rng, n, other, k)
    id_map = np.full(other, -1, np.int32)
    id_map[rng.permutation(other)[:20000]] = rng.permutation(v)[:20000]
    ids[3, 5], ids[4, 6], id_map[ids[5, 0]] = -1, other, v  # outside the map; a map's entry outside the vocabulary
    id_map[ids[6, 1]] = id_map[ids[6, 2]] = 77  # two of the teacher's tokens are one of the student's
    assert split("distill", n, v, dtype, k)
    check(ur.placed(x, dtype, pad=3), ids, lp, (0.5 + rng.random(n)).astype(np.float32), tail, rng.standard_normal(n).astype(np.float32),
          dtype, id_map=id_map)


@pytest.mark.parametrize("dtype", TYPES)
def test_every_kind_of_nan_is_passed_over(dtype):
    rng = np.random.default_rng(37)
    patterns = {"bf16": (0x7F81, 0xFF81, 0x7FC0, 0xFFC1), "f16": (0x7C01, 0xFC01, 0x7E00), "f32": (0x7F800001, -0x7FFFFF, 0x7FC00000)}[dtype]
    n, v, k = 8, WIDE[dtype], 20
    rows = ur.placed(ur.model_rows(rng, n, v), dtype, pad=1)
    bits = rows.view(torch.int32 if dtype == "f32" else torch.int16)
    for i in range(n):
        at = torch.from_numpy(rng.permutation(v)[:rng.integers(1, v)]).cuda()
        pattern = int(patterns[i % len(patterns)])
        bits[i, at] = pattern if dtype == "f32" or pattern < 0x8000 else pattern - 0x10000
    assert rows.isnan().any(1).all() and split("logprobs", n, v, dtype, k) and split("distill", n, v, dtype, k)
    check_logprobs(np.zeros((n, v)), rows, rng.integers(0, v, n), None, k)
    ids, lp = lists(rng, n, v, k)
    check(rows, ids, lp, None, False, rng.standard_normal(n).astype(np.float32), dtype)


def test_rows_of_any_alignment():
    rng = np.random.default_rng(38)
    n, k = 4, 9
    for dtype, v in (("bf16", 65537 + 8), ("f32", 33000)):
        x = ur.model_rows(rng, n, v)
        ids, lp = lists(rng, n, v, k)
        g = rng.standard_normal(n).astype(np.float32)
        assert split("logprobs", n, v, dtype, k) and split("distill", n, v, dtype, k)
        for shift in range(9):
            rows = ur.placed(x, dtype, pad=shift % 3, shift=shift)
            check_logprobs(x, rows, rng.integers(0, v, n), None, k)
            check(rows, ids, lp, None, True, g, dtype, out=ur.placed(x, dtype, pad=(shift + 1) % 3, shift=(shift * 5) % 9))
            check(rows, ids, lp, None, True, g, dtype, out=rows)


