"""Calls of the top logits and the sampling that are refused on the host, before anything
touches a device, beside those of test_answer_abi.py."""
import math

import pytest

from paper_2607_14672_amd import dstd

A = 1 << 40  # made-up addresses, far apart
X, IDX, LOGIT, REST = (A * (k + 1) for k in range(4))


@pytest.mark.parametrize("scale", [2.36e38, -2.36e38, 3e38, -3.4e38])
def test_rest_needs_a_scale_whose_product_with_log2e_fits(scale):
    s = dstd.dstd_scores(X, 4, 100, 100, dstd.DSTD_F32, math.nan, scale)
    assert dstd.dstd_top_logits(s, 5, IDX, LOGIT, REST, None) == dstd.DSTD_ERR_PARAM
    assert "log2" in dstd.dstd_last_error()
    # an empty batch is refused alike
    s = dstd.dstd_scores(None, 0, 100, 100, dstd.DSTD_F32, math.nan, scale)
    assert dstd.dstd_top_logits(s, 5, IDX, LOGIT, REST, None) == dstd.DSTD_ERR_PARAM
