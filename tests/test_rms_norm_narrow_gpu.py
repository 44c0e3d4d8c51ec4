"""RMS norm of rows that a few 16-byte units hold: every value of a row is stored, wherever the row starts, and nothing
besides.  Tolerances: see test_rms_norm_gpu.py."""
import numpy as np
import pytest
import torch

import paper_1501_06633_b200 as mx
from test_rms_norm_gpu import U, norm
from test_train8_gpu import SUM_TOL, WIDE, as_held, data, down, up, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pad", [0, 1, 2, 3, 5])
@pytest.mark.parametrize("cols", [1, 6, 8, 9, 10, 11, 12, 13, 14, 15, 17, 23])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_narrow_rows(cols, pad, kind):
    rng = np.random.default_rng(cols)
    code, tt = WIDE[kind]
    ld = cols + pad
    for rows in (19, 3700):           # read directly, and through the ring
        x, r = as_held(data(rng, rows, cols, False), kind), as_held(data(rng, rows, cols, False) + 0.5, kind)
        d = mx.RmsNormDesc.make(rows, cols, x_type=code, ldx=ld, ldr=ld, ldy=ld)
        s, y, dx = (torch.full((rows, ld), 7.0, dtype=tt, device="cuda") for _ in range(3))
        rstd = torch.empty(rows, device="cuda")
        mx.rms_norm_fprop(d, up(x, tt, ld), residual=up(r, tt, ld), sum=s[:, :cols], y=y[:, :cols], rstd=rstd)
        h = x + r
        want, _ = norm(h, 1.0, 1e-6)
        within(down(s[:, :cols]), h, U * np.abs(h), kind)
        within(down(y[:, :cols]), want, (SUM_TOL + 4 * U) * np.abs(want), kind)
        h = down(s[:, :cols])
        mx.rms_norm_bprop(d, up(r, tt, ld), s[:, :cols], None, rstd, dx[:, :cols])
        k = down(rstd)[:, None]
        hh = h * k
        inner, size = (r * hh).mean(1, keepdims=True), np.abs(r * hh).mean(1, keepdims=True)
        want = k * (r - hh * inner)
        within(down(dx[:, :cols]), want, k * (4 * U * np.abs(r) + np.abs(hh) * (SUM_TOL + 8 * U) * size) + U * np.abs(want), kind)
        for t in (s, y, dx):
            assert bool((t[:, cols:] == 7.0).all())
    assert mx.last_device_status() == mx.OK
