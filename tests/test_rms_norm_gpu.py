"""RMS norm with the residual's addition against its definition in 64 bits.

Tolerances.  x + r is rounded once (2^-24).  The row's sum of squares passes at most 64 additions from a value to the
total, SUM_TOL = 2^-18 of it, and its root half of that; y has three roundings more.  Backward, with rstd given: hh has two
roundings, the row's sum SUM_TOL of the sum of magnitudes, dx four more.  Sums over rows are chains of at most `rows`
additions."""
import numpy as np
import pytest
import torch

import paper_1501_06633_b200 as mx
import train8_ref as ref
from packed_rows import near_rows
from test_train8_gpu import PACKED, SUM_TOL, WIDE, as_held, bytes_of, data, down, up, within

pytestmark = pytest.mark.gpu
U = 2.0 ** -24

# columns: one to several vectors of a lane, odd ones, every number of warps to a row, rows that are read again; rows: a
# few (read directly) and more than the ring's groups
SHAPES = [(1, 1, 0), (2, 7, 0), (5, 64, 0), (3, 1000, 0), (9, 1024, 8), (4, 1025, 3), (6, 2048, 0), (3, 4096, 0), (2, 4100, 0),
          (3, 8192, 0), (2, 9000, 0), (2, 16384, 0), (2, 16392, 0), (2, 20001, 0),
          (7201, 72, 0), (7203, 45, 0), (3701, 520, 0), (3700, 521, 2), (1801, 1032, 0), (901, 2056, 0), (905, 2051, 0),
          (303, 4104, 0), (301, 4101, 0), (299, 8200, 0)]


def norm(h, gamma, eps):
    rstd = 1 / np.sqrt((h * h).mean(1) + eps)
    return h * rstd[:, None] * gamma, rstd


@pytest.mark.parametrize("rows,cols,pad", SHAPES)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_fprop(rows, cols, pad, kind):
    rng = np.random.default_rng(cols)
    code, tt = WIDE[kind]
    x, r = as_held(data(rng, rows, cols, False), kind), as_held(3 * data(rng, rows, cols, False) + 0.5, kind)
    gamma = as_held(rng.uniform(-2, 2, cols), kind)
    ld = cols + pad
    d = mx.RmsNormDesc.make(rows, cols, eps=1e-6, x_type=code, w_type=code, ldx=ld, ldr=ld, ldy=ld)
    tx, tr, g = up(x, tt, ld), up(r, tt, ld), up(gamma, tt)
    s, y = (torch.full((rows, ld), 7.0, dtype=tt, device="cuda") for _ in range(2))
    rstd = torch.empty(rows, device="cuda")
    q, c = mx.empty_packed(rows, cols), mx.empty_packed(rows, cols)
    sq, sc = mx.empty_scales(mx.BLOCK_ROW, rows, cols), mx.empty_scales(mx.BLOCK_ROW, rows, cols)
    mx.rms_norm_fprop(d, tx, g, residual=tr, sum=s[:, :cols], y=y[:, :cols], rstd=rstd, packed=(q, sq), checkpoint=(c, sc))
    h = x + r
    want, wr = norm(h, gamma, 1e-6)
    within(down(s[:, :cols]), h, U * np.abs(h), kind)
    assert np.all(np.abs(down(rstd) - wr) <= SUM_TOL * wr)
    # h's rounding is relative to itself
    tol = (SUM_TOL + 4 * U) * np.abs(want)
    within(down(y[:, :cols]), want, tol, kind)
    assert bool((s[:, cols:] == 7.0).all()) and bool((y[:, cols:] == 7.0).all())
    near_rows(q, sq, want, tol, "e4m3")
    near_rows(c, sc, h, U * np.abs(h), "e4m3")
    # without a residual, every result alone; and the sum in the residual's place
    for name in ("y", "packed", "rstd"):
        y1, r1 = torch.full((rows, ld), 7.0, dtype=tt, device="cuda"), torch.empty(rows, device="cuda")
        q1, s1 = mx.empty_packed(rows, cols), mx.empty_scales(mx.BLOCK_ROW, rows, cols)
        mx.rms_norm_fprop(d, s[:, :cols], g, **{name: {"y": y1[:, :cols], "packed": (q1, s1), "rstd": r1}[name]})
        w1, wr1 = norm(down(s[:, :cols]), gamma, 1e-6)
        if name == "y":
            within(down(y1[:, :cols]), w1, (SUM_TOL + 4 * U) * np.abs(w1), kind)
            assert bool((y1[:, cols:] == 7.0).all())
        elif name == "packed":
            near_rows(q1, s1, w1, (SUM_TOL + 4 * U) * np.abs(w1), "e4m3")
        else:
            assert np.all(np.abs(down(r1) - wr1) <= SUM_TOL * wr1)
    y2, rs2 = torch.empty_like(y), torch.empty_like(rstd)
    mx.rms_norm_fprop(d, tx, g, residual=tr, sum=tr, y=y2[:, :cols], rstd=rs2)
    assert torch.equal(tr, s[:, :cols]) and torch.equal(y2[:, :cols], y[:, :cols]) and torch.equal(rs2, rstd)
    assert mx.last_device_status() == mx.OK


@pytest.mark.parametrize("rows,cols,pad", SHAPES)
@pytest.mark.parametrize("kind,packed", [("f32", None), ("f32", "e5m2"), ("bf16", None), ("bf16", "e4m3"), ("f16", "e4m3"), ("f16", None)])
def test_bprop(rows, cols, pad, kind, packed):
    rng = np.random.default_rng(rows + cols)
    code, tt = WIDE[kind]
    ld = cols + pad
    h = as_held(2.0 * data(rng, rows, cols, False) + 1.0, kind)
    dy, ds = as_held(data(rng, rows, cols, False), kind), as_held(data(rng, rows, cols, False), kind)
    gamma = rng.uniform(-2, 2, cols).astype(np.float32).astype(np.float64)
    rstd = np.float32(norm(h, 1.0, 1e-6)[1]).astype(np.float64)
    if packed:
        # as the library packs it (its packing is compared elsewhere); what it stands for is exact
        th, ts = mx.empty_packed(rows, cols, PACKED[packed][0]), mx.empty_scales(mx.BLOCK_ROW, rows, cols)
        mx.quant8(mx.Quant8Desc.make(rows, cols, x_type=code, q_type=PACKED[packed][0]), up(h, tt), row=(th, ts))
        h = down(th) * np.repeat(ref.value_of(bytes_of(ts)).T, ref.BLOCK, 1)[:, :cols]
        d = mx.RmsNormDesc.make(rows, cols, x_type=PACKED[packed][0], y_type=code, ldx=th.stride(0), ldy=ld, ldr=ld)
    else:
        th, ts = up(h, tt, ld), None
        d = mx.RmsNormDesc.make(rows, cols, x_type=code, ldx=ld, ldy=ld, ldr=ld)
    dx = torch.full((rows, ld), 7.0, dtype=tt, device="cuda")
    dg = torch.empty(cols, device="cuda")
    ws = torch.empty(mx.rms_norm_bprop_workspace(d), dtype=torch.uint8, device="cuda")
    tdy, tds, g, r = up(dy, tt, ld), up(ds, tt, ld), up(gamma, torch.float32), up(rstd, torch.float32)
    mx.rms_norm_bprop(d, tdy, th, g, r, dx[:, :cols], dg, ws, dsum=tds, h_scale=ts)
    hh, e = h * rstd[:, None], dy * gamma
    inner, size = (e * hh).mean(1, keepdims=True), np.abs(e * hh).mean(1, keepdims=True)
    want = rstd[:, None] * (e - hh * inner) + ds
    tol = rstd[:, None] * (4 * U * np.abs(e) + np.abs(hh) * (SUM_TOL + 8 * U) * size) + U * np.abs(want) + 4 * U * np.abs(ds)
    within(down(dx[:, :cols]), want, tol, kind)
    assert bool((dx[:, cols:] == 7.0).all())
    wg, sg = (dy * hh).sum(0), np.abs(dy * hh).sum(0)
    assert np.all(np.abs(down(dg) - wg) <= (rows + 32) * U * sg + 1e-30)
    # neither sums nor dsum; dx in dsum's place
    again = torch.full_like(dx, 7.0)
    mx.rms_norm_bprop(d, tdy, th, g, r, again[:, :cols], h_scale=ts)
    within(down(again[:, :cols]), want - ds, tol, kind)
    mx.rms_norm_bprop(d, tdy, th, g, r, tds, dg, ws, dsum=tds, h_scale=ts)
    assert torch.equal(tds, dx[:, :cols]) and bool((again[:, cols:] == 7.0).all())
    assert mx.last_device_status() == mx.OK


@pytest.mark.parametrize("rows,cols,pad", [(40, 300, 5), (7, 4096, 8), (3, 9000, 3), (400, 2051, 1), (2, 20000, 4)])
def test_bprop_of_packed_rows_of_any_pitch_and_in_place(rows, cols, pad):
    """The packed sum's rows at any place, and dx in dy's memory."""
    gen = torch.Generator(device="cuda").manual_seed(rows)
    h, dy = (torch.randn(rows, cols, device="cuda", generator=gen).to(torch.bfloat16) for _ in range(2))
    q, s = mx.empty_packed(rows, cols), mx.empty_scales(mx.BLOCK_ROW, rows, cols)
    mx.quant8(mx.Quant8Desc.make(rows, cols), h, row=(q, s))
    rstd, dg, dg2 = torch.rand(rows, device="cuda", generator=gen) + 0.5, torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    want = torch.empty_like(dy)
    for ld in (q.stride(0), cols + pad):
        wide = torch.full((rows, ld), 0x7F, dtype=torch.uint8, device="cuda").view(q.dtype)
        wide.view(torch.uint8)[:, :cols] = q.view(torch.uint8)
        d = mx.RmsNormDesc.make(rows, cols, x_type=mx.DTYPE_E4M3, y_type=mx.DTYPE_BF16, ldx=ld)
        ws = torch.empty(mx.rms_norm_bprop_workspace(d), dtype=torch.uint8, device="cuda")
        into = want if ld == q.stride(0) else dy
        mx.rms_norm_bprop(d, dy, wide[:, :cols], None, rstd, into, dg if into is want else dg2, ws, h_scale=s)
    # (the two ways may add the row's sum in another order: half a step of the result, and SUM_TOL of its terms)
    hh = down(q) * np.repeat(ref.value_of(bytes_of(s)).T, ref.BLOCK, 1)[:, :cols] * down(rstd)[:, None]
    assert np.all(np.abs(down(want) - down(dy)) <= 2.0 ** -7 * np.abs(down(want)) + SUM_TOL * down(rstd)[:, None] * (1 + np.abs(hh)) * 8)
    assert float((dg - dg2).abs().max()) <= 1e-4 * float(dg.abs().max())
    assert mx.last_device_status() == mx.OK


def test_gradients_against_differences():
    rows, cols, step = 3, 40, 1e-2
    rng = np.random.default_rng(0)
    x, r, dy, ds = (np.float32(data(rng, rows, cols, False)) for _ in range(4))
    gamma = np.float32(rng.uniform(0.5, 1.5, cols))
    d = mx.RmsNormDesc.make(rows, cols, x_type=mx.DTYPE_F32)
    cuda = lambda a: torch.from_numpy(a).cuda()

    def loss(x, r, gamma):
        y, s = torch.empty(rows, cols, device="cuda"), torch.empty(rows, cols, device="cuda")
        mx.rms_norm_fprop(d, cuda(x), cuda(gamma), residual=cuda(r), sum=s, y=y)
        return float((down(y) * dy).sum() + (down(s) * ds).sum())

    s, rstd = torch.empty(rows, cols, device="cuda"), torch.empty(rows, device="cuda")
    mx.rms_norm_fprop(d, cuda(x), residual=cuda(r), sum=s, rstd=rstd)
    dx, dg = torch.empty(rows, cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(mx.rms_norm_bprop_workspace(d), dtype=torch.uint8, device="cuda")
    mx.rms_norm_bprop(d, cuda(dy), s, cuda(gamma), rstd, dx, dg, ws, dsum=cuda(ds))
    # central differences: step^2 / 6 times a third derivative of a few units; 240 terms rounded in fp32 over 2 step
    tol = 50 * step * step * 0.1 + 1e-5 / (2 * step)
    for grad, of in ((down(dx), 0), (down(dx), 1), (down(dg), 2)):
        for at in rng.choice(grad.size, 12, replace=False):
            args = [x.copy(), r.copy(), gamma.copy()]
            args[of].flat[at] += step
            hi = loss(*args)
            args[of].flat[at] -= 2 * step
            lo = loss(*args)
            assert abs((hi - lo) / (2 * step) - grad.flat[at]) <= tol


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("cols", [96, 100, 4096, 20000])
def test_values_that_are_not_finite_and_rows_of_zeros(kind, cols):
    """A row with a NaN or infinity does not touch its neighbours; a row of zeros is normalised by eps, or gives NaN without."""
    code, tt = WIDE[kind]
    rows = 6
    rng = np.random.default_rng(1)
    x = as_held(rng.standard_normal((rows, cols)), kind)
    x[1, 3], x[3, 5], x[4] = np.nan, np.inf, 0.0
    with np.errstate(invalid="ignore"):
        want, _ = norm(x, 1.0, 1e-6)
    d = mx.RmsNormDesc.make(rows, cols, x_type=code)
    y, q, s = torch.empty(rows, cols, dtype=tt, device="cuda"), mx.empty_packed(rows, cols), mx.empty_scales(mx.BLOCK_ROW, rows, cols)
    mx.rms_norm_fprop(d, up(x, tt), y=y, packed=(q, s))
    got = down(y)
    assert np.isnan(got[1]).all() and np.isnan(got[3, 5]) and np.all(np.delete(got[3], 5) == 0) and np.all(got[4] == 0)
    for r in (0, 2, 5):
        within(got[r], want[r], (SUM_TOL + 4 * U) * np.abs(want[r]), kind)
    near_rows(q[:1], s.view(torch.uint8)[:, :1].contiguous().view(s.dtype), want[:1], (SUM_TOL + 4 * U) * np.abs(want[:1]), "e4m3")
    assert np.isnan(down(q)[1]).all() and np.all(down(q)[4] == 0) and np.all(bytes_of(s)[:, 4] == 127)
    mx.rms_norm_fprop(mx.RmsNormDesc.make(rows, cols, eps=0.0, x_type=code), up(x, tt), y=y)
    assert bool(torch.isnan(y[4]).all()) and not bool(torch.isnan(y[5]).any())


def test_no_rows_and_another_stream():
    d = mx.RmsNormDesc.make(0, 64)
    e = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda")
    dg = torch.full((64,), 5.0, device="cuda")
    mx.rms_norm_fprop(d, e, y=e, rstd=torch.empty(0, device="cuda"))
    mx.rms_norm_bprop(d, e, e, None, torch.empty(0, device="cuda"), torch.empty_like(e), dg)
    assert bool((dg == 0).all())
    x = torch.randn(300, 512, device="cuda")
    d = mx.RmsNormDesc.make(300, 512, x_type=mx.DTYPE_F32)
    want, got = torch.empty_like(x), torch.empty_like(x)
    mx.rms_norm_fprop(d, x, y=want)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    mx.rms_norm_fprop(d, x, y=got, stream=other)
    torch.cuda.current_stream().wait_stream(other)
    assert torch.equal(got, want)


def test_rows_beyond_32_bit_offsets():
    """A matrix of more than 2^31 elements by its pitch: the last row is where its number says."""
    rows, cols, ld = 3, 256, (1 << 30) + 64
    flat = torch.zeros((rows - 1) * ld + cols, dtype=torch.bfloat16, device="cuda")
    x = flat.as_strided((rows, cols), (ld, 1))
    x.copy_(torch.randn(rows, cols, device="cuda"))
    y, dg, dx = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda"), torch.empty(cols, device="cuda"), torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    rstd = torch.empty(rows, device="cuda")
    mx.rms_norm_fprop(mx.RmsNormDesc.make(rows, cols, ldx=ld), x, y=y, rstd=rstd)
    want, _ = norm(down(x.contiguous()), 1.0, 1e-6)
    within(down(y), want, (SUM_TOL + 4 * U) * np.abs(want), "bf16")
    d = mx.RmsNormDesc.make(rows, cols, ldx=ld)
    ws = torch.empty(mx.rms_norm_bprop_workspace(d), dtype=torch.uint8, device="cuda")
    mx.rms_norm_bprop(d, y, x, None, rstd, dx, dg, ws)
    hh = down(x.contiguous()) * down(rstd)[:, None]
    assert np.all(np.abs(down(dg) - (down(y) * hh).sum(0)) <= 40 * U * np.abs(down(y) * hh).sum(0) + 1e-30)
