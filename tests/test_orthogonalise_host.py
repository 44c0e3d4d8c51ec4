"""Refusals and planning of the orthogonalised update, without a GPU."""
import ctypes

import pytest

import paper_1501_06633_b200 as mx
from paper_1501_06633_b200 import train8

P = 4096          # an aligned address that no refused call touches
INVALID, UNSUPPORTED = mx.INVALID_VALUE, mx.NOT_SUPPORTED


def call(desc, x=P, coefficients=None, out=2 * P, ws=3 * P, size=1 << 50):
    return train8._library().maxdnn_orthogonalise(ctypes.byref(desc), x, coefficients, out, ws, size, None)


@pytest.mark.parametrize("fields,status", [
    (dict(batch=-1), INVALID), (dict(rows=0), INVALID), (dict(cols=0), INVALID), (dict(steps=0), INVALID), (dict(steps=33), UNSUPPORTED),
    (dict(x_type=mx.DTYPE_E4M3), INVALID), (dict(x_type=17), INVALID), (dict(ldx=99), INVALID), (dict(ldo=99), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(batch=2, stride_o=6399), INVALID), (dict(batch=2, stride_x=-1), INVALID),
    (dict(rows=65537), UNSUPPORTED), (dict(batch=65537), UNSUPPORTED)])
def test_refusals(fields, status):
    d = mx.OrthoDesc.make(64, 100)
    for k, v in fields.items():
        setattr(d, k, v)
    assert call(d) == status
    n = ctypes.c_size_t()
    assert train8._library().maxdnn_orthogonalise_workspace(ctypes.byref(d), ctypes.byref(n)) == status


def test_missing_and_misaligned():
    d = mx.OrthoDesc.make(64, 100)
    need = mx.orthogonalise_workspace(d)
    for bad in (dict(x=None), dict(x=P + 2), dict(out=None), dict(out=2 * P + 8), dict(ws=None), dict(ws=P + 8), dict(size=need - 1)):
        assert call(d, **bad) == INVALID
    for bad in (float("nan"), float("inf")):
        assert call(d, coefficients=(ctypes.c_float * 15)(*[1.0] * 14, bad)) == INVALID
    assert train8._library().maxdnn_orthogonalise(None, P, None, P, P, 0, None) == INVALID
    assert train8._library().maxdnn_orthogonalise_workspace(ctypes.byref(d), None) == INVALID
    assert call(mx.OrthoDesc.make(64, 100, batch=0), None, None, None, None, 0) == mx.OK


def test_workspace():
    """Four copies of X and two of the shorter side's square in two bytes each, and little besides."""
    for rows, cols, batch in ((4096, 4096, 1), (1000, 2309, 1), (512, 128, 16)):
        n = min(rows, cols)
        least = batch * 2 * (4 * rows * cols + 2 * n * n)
        assert least <= mx.orthogonalise_workspace(mx.OrthoDesc.make(rows, cols, batch=batch)) <= 1.2 * least + 100000


def test_coefficients_are_counted():
    with pytest.raises(ValueError):
        mx.orthogonalise(mx.OrthoDesc.make(8, 8, steps=2), None, None, None, [(1, 2, 3)])
    with pytest.raises(ValueError):
        mx.orthogonalise(mx.OrthoDesc.make(8, 8, steps=2), None, None, None, (1, 2))
