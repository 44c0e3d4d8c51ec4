"""Refusals of the 8-bit training operators and the product's planner, without a GPU: arguments
are checked before the device is."""
import ctypes

import pytest

import paper_1501_06633_b200 as mx
from paper_1501_06633_b200 import train8

P = 4096          # an aligned address that no refused call touches
INVALID, UNSUPPORTED = mx.INVALID_VALUE, mx.NOT_SUPPORTED


def call(name, desc, *args):
    return getattr(train8._library(), name)(ctypes.byref(desc), *args)


def refused(status, name, desc, *args):
    assert call(name, desc, *args) == status


def changed(desc, **fields):
    for k, v in fields.items():
        setattr(desc, k, v)
    return desc


@pytest.mark.parametrize("fields,status", [
    (dict(M=-1), INVALID), (dict(N=-1), INVALID), (dict(K=-1), INVALID), (dict(lda=60), INVALID), (dict(ldb=15), INVALID),
    (dict(ldc=99), INVALID), (dict(a_type=mx.DTYPE_BF16), INVALID), (dict(b_type=9), INVALID), (dict(c_type=mx.DTYPE_E4M3), INVALID),
    (dict(a_major=2), INVALID), (dict(a_block=mx.BLOCK_COL), INVALID), (dict(b_block=3), INVALID),
    (dict(a_scale_type=mx.DTYPE_BF16), INVALID), (dict(lda=72), UNSUPPORTED), (dict(ldb=72), UNSUPPORTED)])
def test_gemm8_refusals(fields, status):
    refused(status, "maxdnn_gemm8", changed(mx.Gemm8Desc.make(10, 100, 64), **fields), P, P, P, P, P, None)


def test_gemm8_null_and_misaligned():
    d = mx.Gemm8Desc.make(10, 100, 64)
    for k in range(5):
        for bad in (None, P + 4):
            if k in (1, 3) and bad:
                continue         # scales are read element by element
            args = [P] * 5
            args[k] = bad
            refused(INVALID, "maxdnn_gemm8", d, *args, None)


@pytest.mark.parametrize("fields,status", [
    (dict(rows=-1), INVALID), (dict(cols=-1), INVALID), (dict(ldx=63), INVALID), (dict(ldq=63), INVALID),
    (dict(x_type=mx.DTYPE_E8M0), INVALID), (dict(q_type=mx.DTYPE_F32), INVALID), (dict(ldq=72), UNSUPPORTED)])
def test_quant8_refusals(fields, status):
    refused(status, "maxdnn_quant8", changed(mx.Quant8Desc.make(10, 64), **fields), P, None, P, P, *[None] * 5)


def test_quant8_missing_parts():
    d = mx.Quant8Desc.make(10, 64)
    refused(INVALID, "maxdnn_quant8", d, P, None, *[None] * 6, None)                     # nothing asked for
    refused(INVALID, "maxdnn_quant8", d, P, None, P, None, *[None] * 4, None)            # values without scales
    refused(INVALID, "maxdnn_quant8", d, P + 2, None, P, P, *[None] * 4, None)
    packed = mx.Quant8Desc.make(10, 64, x_type=mx.DTYPE_E4M3)
    refused(INVALID, "maxdnn_quant8", packed, P, None, P, P, *[None] * 4, None)          # packed x without scales
    refused(INVALID, "maxdnn_dequant8", packed, 0, P, P, P, None)                        # to an 8-bit type
    refused(INVALID, "maxdnn_dequant8", d, 3, P, P, P, None)
    refused(INVALID, "maxdnn_dequant8", d, 0, P, None, P, None)


@pytest.mark.parametrize("fields,status", [
    (dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(ldx=63), INVALID), (dict(ldy=63), INVALID), (dict(eps=-1.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(w_type=mx.DTYPE_E4M3), INVALID), (dict(y_type=mx.DTYPE_E4M3), INVALID),
    (dict(y_type=mx.DTYPE_F32), UNSUPPORTED), (dict(ldq=63), INVALID), (dict(ldq=72), UNSUPPORTED), (dict(q_type=0), INVALID)])
def test_layer_norm_refusals(fields, status):
    refused(status, "maxdnn_layer_norm_fprop", changed(mx.LayerNormDesc.make(10, 64), **fields), P, None, None, P, P, P, P, P, P, P, None)


def test_layer_norm_missing_parts():
    d = mx.LayerNormDesc.make(10, 64)
    refused(INVALID, "maxdnn_layer_norm_fprop", d, P, *[None] * 10)
    refused(INVALID, "maxdnn_layer_norm_fprop", d, P, None, None, None, None, None, P, None, None, None, None)
    refused(INVALID, "maxdnn_layer_norm_bprop", d, P, P, None, None, None, P, P, None, None, None, 0, None)   # no mean
    packed = mx.LayerNormDesc.make(10, 64, x_type=mx.DTYPE_E4M3, y_type=mx.DTYPE_BF16, ldx=64)
    refused(INVALID, "maxdnn_layer_norm_bprop", packed, P, P, None, None, P, P, P, None, None, None, 0, None)
    refused(INVALID, "maxdnn_layer_norm_fprop", packed, P, None, None, P, *[None] * 7)


@pytest.mark.parametrize("fields,status", [
    (dict(rows=-1), INVALID), (dict(cols=-2), INVALID), (dict(ldh=127), INVALID), (dict(lda=63), INVALID), (dict(act=3), INVALID),
    (dict(gated=2), INVALID), (dict(x_type=mx.DTYPE_E4M3), INVALID), (dict(ldq=63), INVALID), (dict(ldc=120), INVALID),
    (dict(ldq=72), UNSUPPORTED), (dict(ldc=136), UNSUPPORTED), (dict(q_type=1), INVALID)])
def test_act8_refusals(fields, status):
    refused(status, "maxdnn_act8_fprop", changed(mx.Act8Desc.make(10, 64), **fields), P, P, P, P, P, P, None)


def test_act8_missing_parts():
    d = mx.Act8Desc.make(10, 64)
    refused(INVALID, "maxdnn_act8_fprop", d, P, *[None] * 6)
    refused(INVALID, "maxdnn_act8_bprop", mx.Act8Desc.make(10, 64, h_type=mx.DTYPE_E4M3), P, P, None, P, None)
    refused(UNSUPPORTED, "maxdnn_act8_bprop", mx.Act8Desc.make(10, 64, h_type=mx.DTYPE_F32), P, P, None, P, None)


def test_null_descriptors():
    lib = train8._library()
    assert lib.maxdnn_gemm8(None, P, P, P, P, P, None) == INVALID
    assert lib.maxdnn_quant8(None, P, *[None] * 8) == INVALID
    assert lib.maxdnn_layer_norm_fprop(None, P, *[None] * 10) == INVALID
    assert lib.maxdnn_act8_fprop(None, P, *[None] * 6) == INVALID


def test_no_rows_is_valid_and_needs_no_device():
    assert call("maxdnn_quant8", mx.Quant8Desc.make(0, 64), *[None] * 9) == mx.OK
    assert call("maxdnn_gemm8", mx.Gemm8Desc.make(0, 8, 64), *[None] * 6) == mx.OK
    assert call("maxdnn_layer_norm_fprop", mx.LayerNormDesc.make(0, 64), *[None] * 11) == mx.OK
    assert call("maxdnn_act8_fprop", mx.Act8Desc.make(0, 64), *[None] * 7) == mx.OK


def test_workspace_grows_with_columns_and_is_bounded_in_rows():
    mx.set_option("SM_COUNT", 148)
    need = lambda r, c: mx.layer_norm_bprop_workspace(mx.LayerNormDesc.make(r, c))
    assert need(1, 4096) == 2 * 4096 * 4
    assert need(10 ** 6, 4096) == need(10 ** 5, 4096)
    assert need(10 ** 6, 20000) > need(10 ** 6, 10000)


def test_binding_checks_tensors():
    import torch
    x = torch.zeros(4, 64)
    with pytest.raises(TypeError):
        mx.layer_norm_fprop(mx.LayerNormDesc.make(4, 64, x_type=mx.DTYPE_F32), x, y=x)
