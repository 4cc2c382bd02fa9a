"""tt.distill against the definition in 64 bits: loss and gradient, with and without the tail, lists of 1 to 128 tokens
with repeated, unmapped and foreign ids, masks, rows without a token or a distribution, in-place gradients, several
groups of rows, streams, graphs; and the operators together as a distillation step uses them."""
import numpy as np
import pytest

import oracle
import util_rows as ur
from gpu_util import to_dev
from test_oracle_logits import bf16_bits

pytestmark = pytest.mark.gpu


def lists(rng, n, width, k, mass=True):
    """Teacher's lists: k tokens a row, descending log probabilities of total 0.5 to 0.98."""
    ids = np.stack([rng.choice(width, k, replace=False) if k <= width else rng.integers(0, width, k) for _ in range(n)]) if n else np.zeros((0, k))
    raw = -1.2 * np.log1p(np.arange(k)) + 0.3 * rng.standard_normal((n, k))
    lp = raw - np.log(np.exp(raw).sum(1, keepdims=True)) + np.log(0.5 + 0.48 * rng.random((n, 1)))
    return ids.astype(np.int32), lp.astype(np.float32)


def check(rows, ids, lp, beta, tail, weight, dtype, id_map=None, out=None, **kw):
    import torch

    import paper_2510_15545_amd as tt

    values = ur.host(rows)
    d = lambda a: None if a is None else to_dev(a)  # noqa: E731
    loss, grad = tt.distill(rows.shape[1], rows, d(ids), d(lp), tail=tail, id_map=d(id_map), inv_temperature=d(beta), grad_loss=d(weight),
                            dlogits=out, **kw)
    torch.cuda.synchronize()
    assert (grad is None) == (weight is None)
    compare(loss, grad, values, ids, lp, beta, tail, weight, dtype, id_map)
    return loss, grad


def compare(loss, grad, values, ids, lp, beta, tail, weight, dtype, id_map=None):
    """The results of rows of these logits against the definition."""
    want, want_d, off, off_d = ur.distill(values, beta, ids, lp, tail, id_map, weight)
    got = ur.host(loss)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want))
    fine = np.isfinite(want)
    bound = (ur.U * np.abs(want) + off)[fine] + 1e-30
    assert np.all(np.abs(got[fine] - want[fine]) <= bound), float((np.abs(got[fine] - want[fine]) / bound).max())
    if grad is None:
        return
    a = ur.host(grad)[:, :values.shape[1]]
    assert np.array_equal(np.isnan(a), np.isnan(want_d))
    fine = np.isfinite(want_d)
    bound = ur.HALF_STEP[dtype] * (np.abs(want_d) + off_d) + off_d + ur.SMALLEST[dtype]
    assert np.all(np.abs(a[fine] - want_d[fine]) <= bound[fine]), float((np.abs(a[fine] - want_d[fine]) / bound[fine]).max())


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("n,v,dtype,k", [(1, 1, "bf16", 1), (2, 2, "f32", 1), (3, 7, "f16", 5), (2, 9, "f32", 9), (4, 640, "bf16", 20),
                                         (3, 4099, "f32", 64), (5, 16385, "bf16", 128), (2, 50257, "f16", 20), (3, 50257, "f32", 33),
                                         (2, 151936, "bf16", 64), (1100, 700, "bf16", 8), (260, 50257, "bf16", 64), (140, 50257, "f32", 16),
                                         (3, 300007, "bf16", 128), (2, 270001, "f32", 20), (257, 20000, "f16", 128), (300, 9001, "bf16", 20), (4, 3001, "f32", 20)])
def test_distill(n, v, dtype, k, tail):
    print(f"[case] distill {n}x{v} {dtype} top {k} tail {tail}", flush=True)
    rng = np.random.default_rng([n, v, k])
    x = ur.model_rows(rng, n, v)
    ids, lp = lists(rng, n, v, k)
    for i in range(n):  # the two models nearly agree
        x[i, ids[i]] = 12.0 + lp[i] + 0.5 * rng.standard_normal(k)
    beta = (0.5 + rng.random(n)).astype(np.float32)
    rows = ur.placed(x, dtype, pad=int(rng.integers(0, 9)), shift=int(rng.integers(0, 9)))
    check(rows, ids, lp, beta, tail, None, dtype)
    check(rows, ids, lp, beta, tail, rng.standard_normal(n).astype(np.float32), dtype)


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_lists_of_every_kind(dtype, tail):
    rng = np.random.default_rng(13)
    n, v, k = 16, 9001, 24
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
    ids[14, 7] = 2 ** 31 - 1
    ids[15, 7] = -2 ** 31
    weight = rng.standard_normal(n).astype(np.float32)
    loss, grad = check(ur.placed(x, dtype, pad=1), ids, lp, None, tail, weight, dtype)
    for i in (3, 4, 6):
        assert ur.host(loss)[i] == 0.0 and not ur.host(grad)[i].any()
    assert np.isnan(ur.host(loss)[9]) and ur.host(loss)[13] == np.inf


@pytest.mark.parametrize("tail", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_masked_and_unsound_rows(dtype, tail):
    rng = np.random.default_rng(14)
    lowest = {"bf16": -3.3895313892515355e38, "f16": -65504.0, "f32": -3.4028234663852886e38}[dtype]
    n, v, k = 18, 5003, 12
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
    beta = np.ones(n, np.float32)
    beta[8:12] = 0.0, -2.0, np.nan, np.inf
    weight = rng.standard_normal(n).astype(np.float32)
    loss, grad = check(ur.placed(x, dtype, pad=2), ids, lp, beta, tail, weight, dtype)
    for i in (1, 2):
        assert ur.host(loss)[i] == 0.0 and not ur.host(grad)[i].any()
    weight[6:12] = 0.0  # padded rows: weight 0 gives zeros whatever the row holds
    _, grad = check(ur.placed(x, dtype, pad=2), ids, lp, beta, tail, weight, dtype)
    assert not ur.host(grad)[6:12].any()


def test_a_list_of_the_whole_vocabulary():
    rng = np.random.default_rng(15)
    for dtype in ("bf16", "f32"):
        for v in (1, 8, 100, 128):
            x = ur.model_rows(rng, 6, v)
            ids, lp = lists(rng, 6, v, v)
            for tail in (False, True):
                check(ur.placed(x, dtype, pad=1), ids, lp, None, tail, np.ones(6, np.float32), dtype)


@pytest.mark.parametrize("tail", [False, True])
def test_lists_of_another_vocabulary(tail):
    rng = np.random.default_rng(16)
    n, v, other, k = 30, 4001, 7003, 50
    x = ur.model_rows(rng, n, v)
    ids, lp = lists(rng, n, other, k)
    id_map = np.full(other, -1, np.int32)
    id_map[rng.permutation(other)[:3000]] = rng.permutation(v)[:3000]
    ids[3, 5], ids[4, 6], id_map[ids[5, 0]] = -1, other, v  # outside the map; a map's entry outside the vocabulary
    id_map[ids[6, 1]] = id_map[ids[6, 2]] = 77  # two of the teacher's tokens are one of the student's
    check(ur.placed(x, "bf16", pad=3), ids, lp, (0.5 + rng.random(n)).astype(np.float32), tail, rng.standard_normal(n).astype(np.float32),
          "bf16", id_map=id_map)


def test_gradient_in_place_and_in_wider_rows():
    import torch

    rng = np.random.default_rng(17)
    n, v, k = 6, 9001, 20
    x = ur.model_rows(rng, n, v)
    ids, lp = lists(rng, n, v, k)
    w = rng.standard_normal(n).astype(np.float32)
    for dtype in ("bf16", "f32"):
        rows = ur.placed(x, dtype, pad=5, shift=2)
        wide = torch.full((n, v + 13), 7.0, dtype=rows.dtype, device="cuda")
        check(rows, ids, lp, None, True, w, dtype, out=wide)
        assert (wide[:, v:] == 7.0).all()  # what lies past v is left alone
        check(rows, ids, lp, None, True, w, dtype, out=rows)


@pytest.mark.parametrize("n,v", [(1205, 262144), (220, 600000)])
def test_many_long_rows(n, v):
    """More rows than are worked on at once, and more split rows than one group holds; in place as well."""
    import torch

    import paper_2510_15545_amd as tt

    rng = np.random.default_rng(18)
    k = 16
    rows = torch.randn((n, v), device="cuda", generator=torch.Generator(device="cuda").manual_seed(5)).mul_(3).bfloat16()
    ids, lp = lists(rng, n, v, k)
    w = rng.standard_normal(n).astype(np.float32)
    args = [to_dev(a) for a in (ids, lp)]
    loss, grad = tt.distill(v, rows, *args, tail=True, grad_loss=to_dev(w))
    some = [0, 1, 73, 110, 111, n - 2, n - 1]
    compare(loss[some], grad[some], ur.host(rows[some]), ids[some], lp[some], None, True, w[some], "bf16")
    again, same = tt.distill(v, rows, *args, tail=True, grad_loss=to_dev(w), dlogits=rows)
    assert torch.equal(again, loss) and torch.equal(same, grad)


def test_streams_and_workspaces_of_the_caller():
    import torch

    import paper_2510_15545_amd as tt

    rng = np.random.default_rng(19)
    n, v, k = 9, 70001, 32  # rows that are split where there are few
    rows = [ur.placed(ur.model_rows(rng, n, v), "bf16") for _ in range(2)]
    ids, lp = (to_dev(a) for a in lists(rng, n, v, k))
    w = torch.ones(n, device="cuda")
    want = [tt.distill(v, r, ids, lp, tail=True, grad_loss=w) for r in rows]
    side = [torch.cuda.Stream() for _ in range(2)]
    spaces = [tt.distill_workspace(n, v, r.dtype, k, grad=True) for r in rows]
    torch.cuda.synchronize()
    for _ in range(4):
        got = [tt.distill(v, r, ids, lp, tail=True, grad_loss=w, stream=s, workspace=ws) for r, s, ws in zip(rows, side, spaces)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    with pytest.raises(tt.TTError):
        tt.distill(v, rows[0], ids, lp, grad_loss=w, workspace=spaces[0][:-256])


def test_replayed_in_a_graph_on_new_inputs():
    import torch

    import paper_2510_15545_amd as tt

    rng = np.random.default_rng(20)
    n, v, k = 9, 20011, 32
    rows = ur.placed(ur.model_rows(rng, n, v), "f16")
    ids, lp = (to_dev(a) for a in lists(rng, n, v, k))
    w = torch.randn(n, device="cuda")
    call = lambda: tt.distill(v, rows, ids, lp, tail=True, grad_loss=w)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for i in range(4):
        rows.copy_(torch.from_numpy(ur.model_rows(rng, n, v)))
        new_ids, new_lp = lists(rng, n, v, k)
        ids.copy_(torch.from_numpy(new_ids))
        lp.copy_(torch.from_numpy(new_lp))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, call())), i


def test_a_distillation_step_across_two_vocabularies():
    """The target's rows give its top tokens (and the log-sum-exp that its verification takes), the vocabularies'
    intersection maps them to the draft's, the draft's rows get their loss and gradient, which goes on through torch."""
    import torch

    import paper_2510_15545_amd as tt
    from paper_2510_15545_amd import synth

    rng = np.random.default_rng(21)
    a = synth.make_vocab(6000, synth.PRINTABLE, 4, [1, 2])
    b = synth.make_vocab(9000, synth.PRINTABLE, 4, [3, 4])
    vd, vt = (tt.Vocab.from_host(x.data, x.offsets, x.max_len) for x in (a, b))
    d2t, t2d = tt.vocab_intersection(vd, tt.token_index(vd), vt, tt.token_index(vt))
    assert int((t2d >= 0).sum()) > 500
    n, k, width = 40, 48, 64
    beta = np.full(n, 0.8, np.float32)
    teacher = ur.placed(ur.model_rows(rng, n, vt.n_tokens), "bf16")
    top = tt.logprobs(vt.n_tokens, teacher, inv_temperature=to_dev(beta), n_top=k)
    hidden = torch.randn((n, width), device="cuda", dtype=torch.float32)
    head = (torch.randn((vd.n_tokens, width), device="cuda") * 0.3).requires_grad_()
    logits = hidden @ head.t()
    weight = torch.full((n,), 1.0 / n, device="cuda")
    loss, grad = tt.distill(vd.n_tokens, logits.detach(), top.top_ids, top.top_logprobs, tail=True, id_map=t2d,
                            inv_temperature=to_dev(beta), grad_loss=weight)
    logits.backward(grad)
    want, want_d, off, off_d = ur.distill(ur.host(logits), beta, top.top_ids.cpu().numpy(), top.top_logprobs.cpu().numpy(), True,
                                          t2d.cpu().numpy(), ur.host(weight))
    assert np.all(np.abs(ur.host(loss) - want) <= off + ur.U * np.abs(want))
    # the head's gradient: sums of n products of fp32, each of the two factors and the sum off by a step a term
    want_head = want_d.T @ ur.host(hidden)
    size = np.abs(want_d.T) @ np.abs(ur.host(hidden))
    assert np.all(np.abs(ur.host(head.grad) - want_head) <= (off_d.T @ np.abs(ur.host(hidden))) + (n + 4) * 2 * ur.U * size + 1e-30)

    # the same rows' log-sum-exp, as verification takes it: 10 streams of 3 proposals
    v, off_ = vt.n_tokens, (np.arange(11) * 3).astype(np.int32)
    ids, q = rng.integers(0, v, 30).astype(np.int32), (rng.random(30) * 1e-3).astype(np.float32)
    ids[::2] = ur.host(teacher)[:, :].argmax(1)[[i for i in range(40) if i % 4 != 3]][::2]
    ua, us = rng.random(30).astype(np.float32), rng.random(10).astype(np.float32)
    nacc, tok = tt.verify_logits(v, to_dev(ids), to_dev(off_), to_dev(q), teacher, to_dev(beta[:10]), to_dev(ua), to_dev(us), 3, lse=top.lse)
    bits = bf16_bits(ur.host(teacher).astype(np.float32))
    o_nacc, o_tok, _ = oracle.verify_logits(v, ids, off_, q, bits, beta[:10], ua, us, max_m=3, lse=top.lse.cpu().numpy())
    assert np.array_equal(nacc.cpu().numpy(), o_nacc) and np.array_equal(tok.cpu().numpy(), o_tok)
    assert 0 < (o_nacc > 0).sum()
