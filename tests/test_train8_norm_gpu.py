"""Layer norm where its sums and differences are delicate: rows far from zero, statistics whose product leaves
the range, values that are not finite.

Tolerances.  Backward, with the statistics given: x - mean is one rounding (a packed x is an exact number) and
its product with rstd another, 2^-23 of xh; a sum over few rows adds one rounding each.  The row sums of
the layer norm pass at most 64 additions from a value to the total, 2^-18 of the sum of magnitudes."""
import numpy as np
import pytest
import torch

import paper_1501_06633_b200 as mx
import train8_ref as ref
from test_train8_gpu import PACKED, SUM_TOL, WIDE, as_held, down, packed_up, up, within

pytestmark = pytest.mark.gpu

# columns of every backward instance: a warp per row (whole and odd), a CTA per row (odd), the ring of 4, 8 and
# 16 warps (with and without columns past the end), rows that are read again
WIDTHS = [64, 300, 301, 512, 1024, 1500, 1501, 2048, 3000, 4096, 4099, 6000, 8192, 8195, 9000]


@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("kind,packed", [("f32", None), ("f32", "e4m3"), ("bf16", "e5m2"), ("f16", None)])
def test_backward_far_from_zero(cols, kind, packed):
    """Rows around 1000 with a spread of 1."""
    rows = 2
    rng = np.random.default_rng(cols)
    x = as_held(1000 + rng.standard_normal((rows, cols)), kind)
    code, tt = WIDE[kind]
    if packed:
        q, s = ref.pack(x, "row", packed)
        x = q * ref.spread(ref.value_of(s), "row", rows, cols)
        t, ts = packed_up(q, s, packed)
        d = mx.LayerNormDesc.make(rows, cols, x_type=PACKED[packed][0], y_type=code, ldx=t.stride(0))
    else:
        t, ts = up(x, tt), None
        d = mx.LayerNormDesc.make(rows, cols, x_type=code)
    # statistics as a forward pass over the unpacked rows would give them
    mean = np.float32(1000 + 0.1 * rng.standard_normal(rows)).astype(np.float64)
    rstd = np.float32(1 + 0.1 * rng.standard_normal(rows)).astype(np.float64)
    dy, gamma = as_held(rng.standard_normal((rows, cols)), kind), np.float32(rng.uniform(0.5, 2, cols)).astype(np.float64)
    dx, dg, db = torch.empty(rows, cols, dtype=tt, device="cuda"), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(mx.layer_norm_bprop_workspace(d), dtype=torch.uint8, device="cuda")
    g, m, r = (up(v, torch.float32) for v in (gamma, mean, rstd))
    mx.layer_norm_bprop(d, up(dy, tt), t, g, m, r, dx, dg, db, ws, x_scale=ts)
    want, wg, wb = ref.layer_norm_grads(x, dy, gamma, mean, rstd)
    xh = np.abs((x - mean[:, None]) * rstd[:, None])
    assert np.all(np.abs(down(dg) - wg) <= (2.0 ** -23 + (rows + 2) * 2.0 ** -24) * (np.abs(dy) * xh).sum(0))
    assert np.all(np.abs(down(db) - wb) <= (rows + 2) * 2.0 ** -24 * np.abs(dy).sum(0))
    e = np.abs(dy * gamma)
    tol = rstd[:, None] * SUM_TOL * (e + e.mean(1, keepdims=True) + xh * (e * xh).mean(1, keepdims=True))
    within(down(dx), want, tol, kind)


@pytest.mark.parametrize("cols", [100, 264, 1000, 1100, 2100, 5000, 9000])
def test_backward_of_equal_values_whose_mean_times_rstd_is_no_number(cols):
    """A row of 1e37 has xh = 0 and rstd = eps^-1/2; what is beyond the row's end takes no part."""
    rows, rstd = 3, np.float32(1 / np.sqrt(1e-5))
    rng = np.random.default_rng(cols)
    x = torch.full((rows, cols), 1e37, device="cuda")
    dy = as_held(rng.standard_normal((rows, cols)), "f32")
    d = mx.LayerNormDesc.make(rows, cols, x_type=mx.DTYPE_F32)
    dx, dg, db = torch.empty(rows, cols, device="cuda"), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(mx.layer_norm_bprop_workspace(d), dtype=torch.uint8, device="cuda")
    m = x[:, 0].contiguous()
    mx.layer_norm_bprop(d, up(dy, torch.float32), x, None, m, torch.full((rows,), float(rstd), device="cuda"), dx, dg, db, ws)
    want = float(rstd) * (dy - dy.mean(1, keepdims=True))
    assert np.all(np.abs(down(dx) - want) <= SUM_TOL * float(rstd) * (np.abs(dy) + np.abs(dy).mean(1, keepdims=True)))
    assert bool((dg == 0).all())
