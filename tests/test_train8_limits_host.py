"""Sizes at the ends of what the 8-bit operators' descriptors can say, without a GPU."""
import ctypes

import pytest

import paper_1501_06633_b200 as mx
from paper_1501_06633_b200 import train8

P = 4096
MOST = 2 ** 31 - 1


def test_layer_norm_of_rows_too_long_for_its_column_numbers():
    """Column numbers are 32 bits: a row is at most 2^30 columns, as in the other operators."""
    lib = train8._library()
    need = ctypes.c_size_t()
    for cols in (MOST, MOST - 6, 2 ** 31 - 8192, 2 ** 30 + 1):
        d = mx.LayerNormDesc.make(2, cols)
        assert lib.maxdnn_layer_norm_fprop(ctypes.byref(d), P, None, None, P, P, P, P, P, P, P, None) == mx.NOT_SUPPORTED
        assert lib.maxdnn_layer_norm_bprop(ctypes.byref(d), P, P, None, None, P, P, P, None, None, None, 0, None) == mx.NOT_SUPPORTED
        assert lib.maxdnn_layer_norm_bprop_workspace(ctypes.byref(d), ctypes.byref(need)) == mx.NOT_SUPPORTED


def test_layer_norm_workspace_of_the_longest_rows():
    mx.set_option("SM_COUNT", 148)
    assert mx.layer_norm_bprop_workspace(mx.LayerNormDesc.make(1000, 2 ** 30)) == 148 * 2 * 2 ** 30 * 4
