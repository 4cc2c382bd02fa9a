"""The calls on rows of logits where they take several launches, or leave the size that caches hold: more rows than one
launch's workgroups, gradients beyond the Infinity Cache's size."""
import numpy as np
import pytest

import util_rows as ur
from test_gpu_distill import compare as compare_distill
from test_gpu_logprobs import compare_logprobs

pytestmark = pytest.mark.gpu

LAUNCH = 1 << 18  # workgroups of one launch


def test_more_rows_than_one_launch_takes():
    """2^18 + 5 rows, a workgroup each: those on both sides of the launches' border are what calls on them alone give."""
    import torch

    import paper_2510_15545_amd as tt

    n, v, k = LAUNCH + 5, 43, 6
    gen = torch.Generator(device="cuda").manual_seed(2)
    rows = torch.randn((n, v), device="cuda", generator=gen).mul_(3).bfloat16()
    ids = torch.randint(0, v, (n,), device="cuda", generator=gen, dtype=torch.int32)
    step = torch.randint(1, 7, (n, 1), device="cuda", generator=gen)
    lists = ((ids[:, None] + step * torch.arange(k, device="cuda")) % v).int()  # different tokens: 7 k < v
    lp = torch.randn((n, k), device="cuda", generator=gen) - 3
    beta = 0.5 + torch.rand(n, device="cuda", generator=gen)
    g, h = (torch.randn(n, device="cuda", generator=gen) for _ in range(2))

    def calls(a, b):
        f = tt.logprobs(v, rows[a:b], ids[a:b], inv_temperature=beta[a:b], n_top=k, entropy=True)
        d = tt.logprobs_backward(v, rows[a:b], ids[a:b], f.stats, g[a:b], entropy=f.entropy, grad_entropy=h[a:b], inv_temperature=beta[a:b])
        return f, d, tt.distill(v, rows[a:b], lists[a:b], lp[a:b], tail=True, inv_temperature=beta[a:b], grad_loss=g[a:b])

    f, d, (loss, grad) = calls(0, n)
    for a, b in ((0, 300), (LAUNCH // 2 - 100, LAUNCH // 2 + 200), (LAUNCH - 200, n)):
        few, few_d, (few_loss, few_grad) = calls(a, b)
        assert all(torch.equal(x[a:b], y) for x, y in zip(f, few)), (a, b)
        assert torch.equal(d[a:b], few_d) and torch.equal(loss[a:b], few_loss) and torch.equal(grad[a:b], few_grad), (a, b)
    some = [0, LAUNCH // 2, LAUNCH - 1, LAUNCH, n - 1]
    host = lambda t: t[some].cpu().numpy()  # noqa: E731
    values = ur.host(rows[some])
    compare_logprobs(ur.logprobs(values, host(ids), host(beta), k), tt.LogProbs(*(t[some] for t in f)))
    compare_distill(loss[some], grad[some], values, host(lists), host(lp), host(beta), True, host(g), "bf16")


@pytest.mark.parametrize("n,v,dtype", [(1100, 128256, "bf16"), (520, 151936, "f32")])
def test_gradients_past_the_cache(n, v, dtype):
    """Over 256 MB of gradients, in memory of their own and in the logits'."""
    import torch

    import paper_2510_15545_amd as tt

    print(f"[case] gradient {n}x{v} {dtype}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(3)
    rows = torch.randn((n, v), device="cuda", generator=gen).mul_(3).to(ur.torch_type(dtype))
    ids = rows.argmax(1).int()
    g, h = (torch.randn(n, device="cuda", generator=gen) for _ in range(2))
    f = tt.logprobs(v, rows, ids, entropy=True)
    some = [0, 1, n // 2, n - 1]
    host = lambda t: t[some].cpu().numpy()  # noqa: E731
    values = ur.host(rows[some])
    got = tt.logprobs_backward(v, rows, ids, f.stats, g, entropy=f.entropy, grad_entropy=h)
    want, off = ur.logprobs_gradient(values, host(ids), None, host(g), host(h))
    bound = ur.HALF_STEP[dtype] * (np.abs(want) + off) + off + ur.SMALLEST[dtype]
    assert np.all(np.abs(ur.host(got[some]) - want) <= bound)
    assert torch.equal(tt.logprobs_backward(v, rows, ids, f.stats, g, entropy=f.entropy, grad_entropy=h, out=rows), got)
