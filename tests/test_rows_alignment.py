"""Layouts of the arrays of the calls on rows of logits: those not aligned to their elements are refused, rows of one
column have any stride between columns."""
import pytest
import torch

import paper_2510_15545_amd as tt
from test_rows_abi import PTR, backward, distill, fake, logprobs


@pytest.mark.parametrize("call,arrays,given", [
    (logprobs, ("temp", "ids", "logprob", "lse", "stats", "entropy", "top_ids", "top_lp"), {}),
    (backward, ("temp", "ids", "stats", "entropy", "g", "h"), dict(entropy=PTR, h=PTR)),
    (distill, ("temp", "ids", "lp", "id_map", "loss", "g"), dict(n_map=5))])
@pytest.mark.parametrize("off", [1, 2, 3])
def test_arrays_off_their_elements(call, arrays, given, off):
    # (100 logits of 200 bytes: rows are whole, the workspace is not looked at)
    for name in arrays:
        assert call(**{**given, name: PTR + off}) == tt.TT_EINVAL, name


def test_one_column_at_any_stride():
    """A row's only element has no next one: what torch calls contiguous may have any stride there."""
    row = torch.zeros(1, 5).t()
    assert row.is_contiguous() and row.stride() == (1, 5)
    assert tt._rows(fake(shape=(5, 1), strides=(1, 5)), 1, 5, "logits") == (0, PTR, 1)
    assert tt._rows(fake(shape=(5, 1), strides=(3, 7), dtype=torch.float32), 1, 5, "logits") == (2, PTR, 3)
    with pytest.raises(ValueError, match="row-major"):
        tt._rows(fake(shape=(5, 2), strides=(1, 5)), 1, 5, "logits")
    with pytest.raises(ValueError, match="at least"):
        tt._rows(fake(shape=(5, 1), strides=(1, 5)), 2, 5, "logits")


@pytest.mark.gpu
def test_one_token_in_all():
    x = torch.randn(1, 5, device="cuda")
    ids, ones = torch.zeros(5, dtype=torch.int32, device="cuda"), torch.ones(5, device="cuda")
    f = tt.logprobs(1, x.t(), ids, n_top=1, entropy=True)
    assert torch.equal(f.lse, x[0]) and not f.logprob.any() and not f.entropy.any() and not f.top_ids.any()
    assert not tt.logprobs_backward(1, x.t(), ids, f.stats, ones).any()
    loss, grad = tt.distill(1, x.t(), ids[:, None], f.logprob[:, None], grad_loss=ones)
    assert not loss.any() and not grad.any()
