"""tt_quantize_i8 on more rows than one launch takes."""
import pytest
import torch

import paper_2510_15545_amd as tt
import util_head as uh
from test_gpu_i8 import definition

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,k,name", [((1 << 22) + 5, 3, "f32"), ((1 << 20) + 3, 4100, "bf16"), ((1 << 26) + 5, 3, "bf16")])
def test_quantize_many_rows(n, k, name):
    """Groups of weights quantised for themselves: the same 1,021 rows over and over, each as by itself; what lies behind is left alone."""
    some = (torch.randn((1021, k), generator=torch.Generator().manual_seed(k)) * torch.logspace(-3, 2, 1021)[:, None]).to(uh.TYPES[name]).cuda()
    times = n // 1021 + 1
    x = some.repeat(times, 1)[:n]
    q, scale = torch.full((n + 2, k), 5, dtype=torch.int8, device="cuda"), torch.full((n + 2,), 5.0, device="cuda")
    tt.quantize_i8(x, out=(q[:n], scale[:n]))
    want_q, want_scale = definition(some)
    assert torch.equal(q[:n], want_q.repeat(times, 1)[:n]) and torch.equal(scale[:n], want_scale.repeat(times)[:n])
    assert bool((q[n:] == 5).all()) and bool((scale[n:] == 5.0).all())
