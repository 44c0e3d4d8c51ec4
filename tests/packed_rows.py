"""Comparison of matrices packed in rows with 64-bit values, without a loop over the blocks."""
import numpy as np

import train8_ref as ref
from test_train8_gpu import bytes_of, down


def near_rows(q, s, x, tol, kind):
    """q, s (row blocks) hold x: within half a step of the 8-bit type, and tol; the scales are the least that hold their block."""
    top, bits, least, _ = ref.SPEC[kind]
    rows, cols = x.shape
    pad = ((0, 0), (0, -cols % ref.BLOCK))
    scale = ref.value_of(bytes_of(s)).T                       # [row][block]
    each = np.repeat(scale, ref.BLOCK, 1)[:, :cols]
    m = np.maximum(np.abs(x), 2.0 ** least * each)
    half = np.ldexp(1.0, np.frexp(m)[1] - bits - 2)
    assert np.all(np.abs(down(q) * each - x) <= half * 1.0001 + tol)
    cut = lambda a: np.pad(a, pad).reshape(rows, -1, ref.BLOCK).max(2)
    peak, slack = cut(np.abs(x)), cut(tol)
    ok = (top * scale >= peak - slack) & ((top * scale / 2 <= peak + slack) | (scale == 2.0 ** -126))
    assert np.all(ok | (peak <= slack))
