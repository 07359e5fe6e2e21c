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


def test_make_scores_refuses_what_the_kernels_cannot_read():
    """A struct of a CPU tensor's address would be read on the GPU, one of another type as
    bf16, one without dimensions not at all."""
    import torch
    with pytest.raises(ValueError, match="GPU"):
        dstd.make_scores(torch.zeros(4, 9))
    with pytest.raises(TypeError, match="float32"):
        dstd.make_scores(torch.zeros(4, 9, dtype=torch.float16))
    with pytest.raises(TypeError, match="tensor"):
        dstd.make_scores([[1.0, 2.0]])


@pytest.mark.gpu
def test_make_scores_refuses_rows_that_are_not_whole():
    import torch
    x = torch.zeros(30, 20, device="cuda")
    for bad in (x.t(), x[:, ::2], x[:1].expand(4, 20), x.as_strided((5, 20), (10, 1))):
        with pytest.raises(ValueError, match="whole"):
            dstd.make_scores(bad)
    with pytest.raises(ValueError, match="dimensions"):
        dstd.make_scores(x[0])
    for good, ld in ((x, 20), (x[::3], 60), (x[:, 3:9], 20), (x[4:5, 2:], 18)):
        s = dstd.make_scores(good)
        assert (s.x, s.B, s.N, s.ld) == (good.data_ptr(), *good.shape, ld)
