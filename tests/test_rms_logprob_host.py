"""Refusals of the RMS norm and the log probabilities, without a GPU: arguments are checked before the device is."""
import ctypes

import pytest

import paper_1501_06633_b200 as mx
from paper_1501_06633_b200 import train8

P = 4096          # an aligned address that no refused call touches
INVALID, UNSUPPORTED = mx.INVALID_VALUE, mx.NOT_SUPPORTED
MOST = 2 ** 31 - 1


def call(name, desc, *args):
    return getattr(train8._library(), "maxdnn_" + name)(ctypes.byref(desc), *args)


def changed(desc, **fields):
    for k, v in fields.items():
        setattr(desc, k, v)
    return desc


FPROP = (P, P, P, P, 2 * P, P, P, P, P, P, None)          # x residual gamma sum y rstd q s c sc stream
BPROP = (P, P, None, P, P, P, 2 * P, P, P, 1 << 40, None)  # dy h scale gamma rstd dsum dx dgamma workspace bytes stream


@pytest.mark.parametrize("fields,status", [
    (dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(ldx=63), INVALID), (dict(ldy=63), INVALID), (dict(ldr=63), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(w_type=mx.DTYPE_E4M3), INVALID), (dict(x_type=9), INVALID),
    (dict(y_type=mx.DTYPE_E4M3), INVALID), (dict(y_type=mx.DTYPE_F32), UNSUPPORTED), (dict(ldq=63), INVALID), (dict(ldq=72), UNSUPPORTED),
    (dict(q_type=0), INVALID), (dict(cols=MOST, ldx=MOST, ldy=MOST, ldr=MOST), UNSUPPORTED)])
def test_rms_norm_refusals(fields, status):
    assert call("rms_norm_fprop", changed(mx.RmsNormDesc.make(10, 64), **fields), *FPROP) == status
    if not set(fields) & {"ldq", "q_type"}:
        assert call("rms_norm_bprop", changed(mx.RmsNormDesc.make(10, 64), **fields), *BPROP) == status


def test_rms_norm_missing_and_misaligned():
    d = mx.RmsNormDesc.make(10, 64)
    put = lambda base, at, v: base[:at] + (v,) + base[at + 1:]
    assert call("rms_norm_fprop", d, P, *[None] * 10) == INVALID                    # nothing asked for
    for at, v in ((0, None), (0, P + 2), (1, P + 8), (3, P + 2), (4, P + 4), (6, P + 1), (7, None), (8, P + 1), (9, None)):
        assert call("rms_norm_fprop", d, *put(FPROP, at, v)) == INVALID
    for at, v in ((0, None), (0, P + 2), (1, None), (1, P + 8), (4, None), (5, P + 2), (6, None), (6, P + 2), (6, P), (8, None), (8, P + 4), (9, 0)):
        if (at, v) in ((8, None), (8, P + 4), (9, 0)):
            continue                                                                # (planned for the device: test_rms_norm_gpu.py)
        assert call("rms_norm_bprop", d, *put(BPROP, at, v)) == INVALID
    packed = mx.RmsNormDesc.make(10, 64, x_type=mx.DTYPE_E4M3, y_type=mx.DTYPE_BF16)
    assert call("rms_norm_bprop", packed, *BPROP) == INVALID                        # packed h without scales
    assert call("rms_norm_fprop", packed, *FPROP) == INVALID
    # the sum may take x's place only with x's pitch, dx dsum's only with dsum's
    assert call("rms_norm_fprop", mx.RmsNormDesc.make(10, 64, ldx=80), P, 2 * P, None, P, *[None] * 7) == INVALID
    assert call("rms_norm_bprop", mx.RmsNormDesc.make(10, 64, ldr=80), P, 3 * P, None, P, P, 2 * P, 2 * P, None, None, 0, None) == INVALID


def test_rms_norm_workspace_is_bounded_in_rows():
    mx.set_option("SM_COUNT", 148)
    need = lambda r, c, **k: mx.rms_norm_bprop_workspace(mx.RmsNormDesc.make(r, c, **k))
    assert need(1, 4096) == 4096 * 4
    assert need(10 ** 6, 4096) == need(10 ** 5, 4096) > need(100, 4096)
    assert need(1000, 2 ** 30) == 148 * 2 ** 30 * 4


FWD = (P, P, P, P, P, P, P, None)                          # x target logprob lse entropy top_logprob top_index stream
BWD = (P, P, P, P, P, P, 2 * P, P, P, P, P, None)          # x target lse dlogprob entropy dentropy dx q_row s_row q_col s_col stream


@pytest.mark.parametrize("fields,status", [
    (dict(rows=-1), INVALID), (dict(cols=0), INVALID), (dict(ldx=99), INVALID), (dict(x_type=mx.DTYPE_E4M3), INVALID), (dict(top=-1), INVALID),
    (dict(top=33), UNSUPPORTED), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(target_type=2), INVALID), (dict(cols=MOST, ldx=MOST, ldd=MOST, ldq=2 ** 31), UNSUPPORTED),
    (dict(rows=MOST), UNSUPPORTED), (dict(rows=2 ** 30 + 1), UNSUPPORTED)])
def test_logprob_refusals(fields, status):
    assert call("logprob_fprop", changed(mx.LogprobDesc.make(10, 100, top=3), **fields), *FWD) == status
    assert call("logprob_bprop", changed(mx.LogprobDesc.make(10, 100, top=3), **fields), *BWD) == status


@pytest.mark.parametrize("fields,status", [(dict(ldd=99), INVALID), (dict(ldq=96), INVALID), (dict(ldq=104), UNSUPPORTED), (dict(q_type=0), INVALID)])
def test_logprob_gradient_refusals(fields, status):
    assert call("logprob_bprop", changed(mx.LogprobDesc.make(10, 100), **fields), *BWD) == status


def test_logprob_missing_and_misaligned():
    put = lambda base, at, v: base[:at] + (v,) + base[at + 1:]
    d = mx.LogprobDesc.make(10, 100, top=3)
    for at, v in ((0, None), (0, P + 4), (1, None), (1, P + 4)):
        assert call("logprob_fprop", d, *put(FWD, at, v)) == INVALID
    assert call("logprob_fprop", d, P, P, *[None] * 6) == INVALID                   # nothing asked for
    assert call("logprob_fprop", mx.LogprobDesc.make(10, 100), *FWD) == INVALID     # alternatives, but none of them
    for at, v in ((0, None), (0, P + 4), (1, None), (1, P + 4), (2, None), (4, None), (6, P), (6, P + 2), (7, P + 1), (8, None), (9, P + 8), (10, None)):
        assert call("logprob_bprop", d, *put(BWD, at, v)) == INVALID
    assert call("logprob_bprop", d, P, P, P, None, P, None, P, *[None] * 5) == INVALID       # no gradient given
    assert call("logprob_bprop", d, P, P, P, P, P, P, None, *[None] * 5) == INVALID          # nothing asked for
    assert call("logprob_bprop", mx.LogprobDesc.make(10, 100, ldd=112), P, P, P, P, P, P, P, *[None] * 5) == INVALID   # in place, other pitch


def test_no_rows_and_null_descriptors():
    lib = train8._library()
    assert call("rms_norm_fprop", mx.RmsNormDesc.make(0, 64), *[None] * 11) == mx.OK
    assert call("logprob_fprop", mx.LogprobDesc.make(0, 64), *[None] * 8) == mx.OK
    assert call("logprob_bprop", mx.LogprobDesc.make(0, 64), *[None] * 12) == mx.OK
    assert lib.maxdnn_rms_norm_fprop(None, *FPROP) == INVALID
    assert lib.maxdnn_rms_norm_bprop(None, *BPROP) == INVALID
    assert lib.maxdnn_rms_norm_bprop_workspace(None, None) == INVALID
    assert lib.maxdnn_logprob_fprop(None, *FWD) == INVALID
    assert lib.maxdnn_logprob_bprop(None, *BWD) == INVALID


def test_binding_checks_tensors():
    import torch
    x = torch.zeros(4, 64)
    with pytest.raises(TypeError):
        mx.rms_norm_fprop(mx.RmsNormDesc.make(4, 64, x_type=mx.DTYPE_F32), x, y=x)
    with pytest.raises(TypeError):
        mx.logprob_fprop(mx.LogprobDesc.make(4, 64, x_type=mx.DTYPE_F32), x, lse=x[:, 0])
