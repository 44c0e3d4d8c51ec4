"""Refusals of values at the ends of their ranges, without a GPU (no rows: an accepted call does nothing)."""
import ctypes

import pytest

import paper_1501_06633_b200 as mx
from paper_1501_06633_b200 import train8


@pytest.mark.parametrize("scale,status", [(1e-45, mx.OK), (1.0, mx.OK), (2.0 ** 127, mx.OK), (1.0000001 * 2.0 ** 127, mx.NOT_SUPPORTED),
                                          (2.4e38, mx.NOT_SUPPORTED), (3.4e38, mx.NOT_SUPPORTED)])
def test_logprob_scales_whose_multiple_of_log2_e_has_no_number(scale, status):
    d = mx.LogprobDesc.make(0, 100, scale=scale)
    lib = train8._library()
    assert lib.maxdnn_logprob_fprop(ctypes.byref(d), *[None] * 8) == status
    assert lib.maxdnn_logprob_bprop(ctypes.byref(d), *[None] * 12) == status
