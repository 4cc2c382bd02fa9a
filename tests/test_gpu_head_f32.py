"""fp32 on the output head: products of fp32 operands in fp32, at long hidden states and vocabularies."""
import pytest
import torch

import paper_2510_15545_amd as tt
import util_head as uh

pytestmark = pytest.mark.gpu


def plain(x, w, ids, stats, g, beta):
    """(logprob, dhidden, dweight) by elementary operations in fp32."""
    z = x @ w.T
    b, at = beta[:, None], ids.long()[:, None]
    top = z.amax(1, keepdim=True)
    y = (z - top) * b
    logprob = (y.gather(1, at) - y.exp().sum(1, keepdim=True).log())[:, 0]
    lp = (z - stats[:, :1]) * b - stats[:, 1:]
    d = -g[:, None] * lp.exp()
    d.scatter_(1, at, -g[:, None] * torch.expm1(lp.gather(1, at)))
    d = d * b
    return logprob, d @ w, d.T.contiguous() @ x


@pytest.mark.parametrize("n,v,h", [(8, 30011, 2048), (40, 5000, 4096), (96, 32000, 512), (70, 20011, 2048), (300, 3001, 1024), (500, 600, 4096)])
def test_no_bits_are_left_out(n, v, h):
    """Relative errors of all values together.  Two orders of the same fp32 roundings (each at most U, or 2 U where the matrix cores
    do not round to nearest) have errors of one size: at most twice that of the elementary operations, and 4 U where those happen to
    have next to none.  Operands rounded to 16 bits of digits are beyond it: 2^-17 of every product's size, 7.6e-6 against under 3e-6."""
    x, w, ids, beta = uh.operands(n, v, h, "f32")
    gen = torch.Generator().manual_seed(n)
    g = (torch.rand(n, generator=gen) + 0.5).cuda()
    got = tt.head_logprobs(v, x, w, ids, inv_temperature=beta)
    grads = tt.head_logprobs_backward(v, x, w, ids, got.stats, g, inv_temperature=beta)
    mine = (got.logprob, *grads)
    want = (uh.forward(x, w, ids, beta)[0]["logprob"], *uh.backward(x, w, ids, uh.forward(x, w, ids, beta)[0]["stats"], g, None, beta)[:2])
    for a, b, c, what in zip(mine, want, plain(x, w, ids, got.stats, g, beta), ("logprob", "dhidden", "dweight")):
        off, theirs = (float((t.double() - b).norm() / b.norm()) for t in (a, c))
        print(f"[case] {n}x{v}x{h} {what}: {off:.2e}, elementary {theirs:.2e}", flush=True)
        assert off <= 2 * theirs + 4 * uh.U, (what, off, theirs)
