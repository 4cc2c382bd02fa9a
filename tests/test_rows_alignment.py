"""Arrays that are not aligned to their elements are refused by the calls on rows of logits."""
import pytest

import paper_2510_15545_amd as tt
from test_rows_abi import PTR, backward, distill, logprobs


@pytest.mark.parametrize("call,arrays,given", [
    (logprobs, ("temp", "ids", "logprob", "lse", "stats", "entropy", "top_ids", "top_lp"), {}),
    (backward, ("temp", "ids", "stats", "entropy", "g", "h"), dict(entropy=PTR, h=PTR)),
    (distill, ("temp", "ids", "lp", "id_map", "loss", "g"), dict(n_map=5))])
@pytest.mark.parametrize("off", [1, 2, 3])
def test_arrays_off_their_elements(call, arrays, given, off):
    # (100 logits of 200 bytes: rows are whole, the workspace is not looked at)
    for name in arrays:
        assert call(**{**given, name: PTR + off}) == tt.TT_EINVAL, name
