"""Which kernels of the sampling the built library holds, by the names it registers: those
that some call launches, and no others."""
import os
import re

import pytest

from paper_2607_14672_amd import build


def test_sampling_holds_no_kernel_that_no_call_launches():
    if not os.path.exists(build.LIB):
        pytest.skip("the library is not built")
    with open(build.LIB, "rb") as f:
        names = set(re.findall(rb"sample_kernelILi(\d+)ELb([01])ELb([01])E([ft])E", f.read()))
    # threads a row, top_k, top_p, type; rows of 64 threads have 512 entries at most, and a
    # top_k of up to 1024 is drawn from a list by other kernels
    want = {(t, k, p, e) for t in (b"64", b"256", b"1024") for k in (b"0", b"1") for p in (b"0", b"1")
            for e in (b"f", b"t") if not (t == b"64" and k == b"1")}
    assert names == want
