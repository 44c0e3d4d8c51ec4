"""Values that are not finite, and scale bytes at the ends of their range: they reach what their formulas say
and nothing else."""
import numpy as np
import pytest
import torch

import paper_1501_06633_b200 as mx
import train8_ref as ref
from test_train8_gpu import ACTS, FORM, PACKED, WIDE, as_held, bytes_of, data, down, packed_up, same, up

pytestmark = pytest.mark.gpu
INF, NAN = np.inf, np.nan


# ------------------------------------------------------------------ product, scales applied by the tensor core
@pytest.mark.parametrize("pair,cols", [(-1, 16), (-1, 32), (-1, 64), (-1, 128), (1, 128), (1, 192), (1, 224), (1, 256)])
@pytest.mark.parametrize("swap", [0, 1])
@pytest.mark.parametrize("ct", ["f32", "bf16"])
def test_product_with_special_values_and_scales(pair, cols, swap, ct):
    """Infinity and NaN among the values, and E8M0 bytes 255 (NaN), 0 (2^-127) and 254 (2^127) on single rows, next to
    rows of ordinary ones."""
    M, N, K = 300, 270, 384
    rng = np.random.default_rng(cols)
    qa, _ = ref.pack(data(rng, M, K, False), "row", "e5m2")
    qb, _ = ref.pack(data(rng, N, K, False), "row", "e4m3")
    qa = np.where(qa == 0, 1.0, qa)
    qb = np.where(qb == 0, 1.0, qb)
    sa = rng.integers(125, 130, (3, M)).astype(np.uint8)
    sb = rng.integers(125, 130, (3, N)).astype(np.uint8)
    qa[5, 7], qa[131, 300], qb[9, 200] = INF, NAN, NAN
    sa[1, 20], sb[2, 258] = 255, 255
    sa[:, 40], sa[:, 170] = 0, 254
    sb[:, 50], sb[:, 200] = 254, 0
    (ta, tsa), (tb, tsb) = packed_up(qa, sa, "e5m2"), packed_up(qb, sb, "e4m3")
    c = torch.empty(M, N, dtype=WIDE[ct][1], device="cuda")
    mx.set_option("GEMM8_PAIR", pair)
    mx.set_option("GEMM8_COLS", cols)
    mx.set_option("GEMM8_SWAP", swap)
    mx.set_option("GEMM8_SPLIT", 1)
    mx.gemm8(mx.Gemm8Desc.make(M, N, K, a_type=mx.DTYPE_E5M2, b_block=mx.BLOCK_ROW, c_type=WIDE[ct][0]), ta, tsa, tb, tsb, c)
    assert mx.last_device_status() == mx.OK
    got = down(c)
    va = qa * ref.spread(2.0 ** (sa.astype(np.float64) - 127), "row", M, K)
    vb = qb * ref.spread(2.0 ** (sb.astype(np.float64) - 127), "row", N, K)
    nan_rows, nan_cols = [20, 131], [9, 258]
    assert np.isnan(got[nan_rows]).all() and np.isnan(got[:, nan_cols]).all()
    plain_cols = np.delete(np.arange(N), nan_cols)
    assert not np.isfinite(got[5, plain_cols]).any()
    rows, cols_ = np.delete(np.arange(M), nan_rows + [5]), plain_cols
    va, vb = va[rows], vb[cols_]
    want, mags = va @ vb.T, np.abs(va) @ np.abs(vb).T
    sub = got[np.ix_(rows, cols_)]
    inside = mags < 2.0 ** 127        # (beyond: sums may leave the range)
    assert inside.sum() > inside.size - 2 * (M + N)
    at = {r: i for i, r in enumerate(rows)}, {n: i for i, n in enumerate(cols_)}
    assert inside[at[0][40], at[1][50]] and inside[at[0][170], at[1][200]]
    # 16-bit: 2^-8 of the value for its rounding (at most half a step of 2^-7); 2^-126 where numbers are subnormal
    tol = (128 + 3) * 2.0 ** -23 * mags + (2.0 ** -8 * np.abs(want) if ct == "bf16" else 0) + 2.0 ** -126
    assert np.all(np.abs(sub - want)[inside] <= tol[inside])


@pytest.mark.parametrize("block", ["row", "col", "tile"])
@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
def test_unpacking_with_scales_at_the_ends(block, kind):
    rows, cols = 130, 260
    rng = np.random.default_rng(2)
    q, s = ref.pack(data(rng, rows, cols), block, kind)
    flat = s.reshape(-1)
    flat[0], flat[1], flat[2] = 0, 254, 255
    s = flat.reshape(s.shape)
    t, ts = packed_up(q, s, kind)
    x = torch.empty(rows, cols, device="cuda")
    mx.dequant8(mx.Quant8Desc.make(rows, cols, x_type=mx.DTYPE_F32, q_type=PACKED[kind][0]), t, ts, x, FORM[block])
    with np.errstate(over="ignore", invalid="ignore"):
        want = q * ref.spread(ref.value_of(s), block, rows, cols)
        same(down(x), as_held(want, "f32"))


# ------------------------------------------------------------------ layer norm
@pytest.mark.parametrize("rows,cols", [(12, 100), (12, 301), (12, 2048), (12, 4096), (700, 384), (700, 1024), (700, 2048), (12, 9000),
                                       (12, 20001)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_layer_norm_rows_that_are_not_finite(rows, cols, kind):
    rng = np.random.default_rng(cols)
    x = as_held(data(rng, rows, cols, False), kind)
    clean = x.copy()
    x[2, 5], x[4, cols - 1], x[7, 90], x[9, 0] = INF, -INF, NAN, INF
    x[9, cols // 2] = -INF
    bad = [2, 4, 7, 9]
    code, tt = WIDE[kind]
    d = mx.LayerNormDesc.make(rows, cols, x_type=code)

    def run(x):
        got = dict(y=torch.zeros(rows, cols, dtype=tt, device="cuda"), mean=torch.zeros(rows, device="cuda"),
                   rstd=torch.zeros(rows, device="cuda"))
        q, c = (mx.empty_packed(rows, cols) for _ in range(2))
        s, sc = (mx.empty_scales(mx.BLOCK_ROW, rows, cols) for _ in range(2))
        mx.layer_norm_fprop(d, up(x, tt), packed=(q, s), checkpoint=(c, sc), **got)
        return dict({k: down(v) for k, v in got.items()}, q=down(q), s=bytes_of(s).T, c=down(c), sc=bytes_of(sc).T)

    got, plain = run(x), run(clean)
    for name in got:
        same(np.delete(got[name], bad, 0), np.delete(plain[name], bad, 0))
    # mean, differences and deviations of such a row are no numbers
    assert np.isnan(got["y"][bad]).all() and np.isnan(got["q"][bad]).all() and np.isnan(got["rstd"][bad]).all()
    assert (got["s"][bad] == 127).all()
    wq, ws = ref.pack(x[bad], "row", "e4m3")
    same(got["c"][bad], wq)
    np.testing.assert_array_equal(got["sc"][bad], ws.T)


@pytest.mark.parametrize("rows,cols", [(12, 100), (12, 301), (12, 1024), (12, 1501), (12, 2048), (12, 4096), (12, 8192), (12, 9000)])
@pytest.mark.parametrize("packed", [False, True])
def test_layer_norm_gradients_that_are_not_finite(rows, cols, packed):
    """A NaN or infinity in dy makes its row of dx and its column of the sums so, one in x its row of dx and its
    column of dgamma; other rows and columns keep their bits."""
    rng = np.random.default_rng(cols)
    x, dy = as_held(data(rng, rows, cols, False), "bf16"), as_held(data(rng, rows, cols, False), "bf16")
    _, mean, rstd = ref.layer_norm(x, 1.0, 0.0, 1e-5)
    d = mx.LayerNormDesc.make(rows, cols)
    ws = torch.empty(mx.layer_norm_bprop_workspace(d) + 4096, dtype=torch.uint8, device="cuda")
    m, r = up(np.float32(mean), torch.float32), up(np.float32(rstd), torch.float32)

    def run(x, dy):
        got = [torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda"), torch.zeros(cols, device="cuda"), torch.zeros(cols, device="cuda")]
        if packed:
            q, s = ref.pack(x, "row", "e5m2")
            t, ts = packed_up(q, s, "e5m2")
            dd = mx.LayerNormDesc.make(rows, cols, x_type=mx.DTYPE_E5M2, y_type=mx.DTYPE_BF16, ldx=t.stride(0))
            mx.layer_norm_bprop(dd, up(dy, torch.bfloat16), t, None, m, r, *got, ws, x_scale=ts)
        else:
            mx.layer_norm_bprop(d, up(dy, torch.bfloat16), up(x, torch.bfloat16), None, m, r, *got, ws)
        return [down(t) for t in got]

    dx0, dg0, db0 = run(x, dy)
    x2, dy2 = x.copy(), dy.copy()
    dy2[2, 5], dy2[6, 40], x2[8, 77] = NAN, INF, NAN
    dx, dg, db = run(x2, dy2)
    bad = [2, 6, 8]
    same(np.delete(dx, bad, 0), np.delete(dx0, bad, 0))
    same(np.delete(dg, [5, 40, 77]), np.delete(dg0, [5, 40, 77]))
    same(np.delete(db, [5, 40]), np.delete(db0, [5, 40]))
    assert np.isnan(dx[[2, 8]]).all() and not np.isfinite(dx[6]).any()
    assert np.isnan(dg[[5, 77]]).all() and not np.isfinite(dg[40]) and np.isnan(db[5]) and db[40] == INF


# ------------------------------------------------------------------ activation
@pytest.mark.parametrize("cols", [128, 300, 301])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("gated", [True, False])
def test_activation_of_values_that_are_not_finite(cols, kind, act, gated):
    """f(inf) = inf; f(-inf) and f(NaN) are NaN (-inf x 0); what is not finite is NaN in E4M3 and touches no
    neighbour's scale."""
    rows, many = 20, 2 if gated else 1
    rng = np.random.default_rng(cols)
    h = as_held(data(rng, rows, many * cols, False), kind)
    clean = h.copy()
    at = {(2, 5): INF, (4, 100): -INF, (6, cols - 1): NAN}
    for (r, c), v in at.items():
        h[r, c] = v
    if gated:
        h[9, cols + 3], h[11, 2 * cols - 1] = INF, NAN
    code, tt = WIDE[kind]
    d = mx.Act8Desc.make(rows, cols, act=ACTS[act], gated=gated, x_type=code)
    db = mx.Act8Desc.make(rows, cols, act=ACTS[act], gated=gated, x_type=code, h_type=mx.DTYPE_E4M3)
    da = as_held(data(rng, rows, cols, False), kind)

    def run(h):
        a, dh, dh8 = (torch.zeros(rows, n * cols, dtype=tt, device="cuda") for n in (1, many, many))
        q, c = mx.empty_packed(rows, cols), mx.empty_packed(rows, many * cols)
        s, sc = mx.empty_scales(mx.BLOCK_ROW, rows, cols), torch.zeros(many * ref.blocks(cols), rows, dtype=torch.uint8, device="cuda")
        th = up(h, tt)
        mx.act8_fprop(d, th, a=a, packed=(q, s), checkpoint=(c, sc))
        mx.act8_bprop(d, up(da, tt), th, dh)
        mx.act8_bprop(db, up(da, tt), c, dh8, h_scale=sc)
        return [down(a), down(q), bytes_of(s), down(c), bytes_of(sc), down(dh), down(dh8)]

    a, q, s, c, sc, dh, dh8 = run(h)
    a0, q0, s0, _, _, dh0, _ = run(clean)
    touched = np.zeros((rows, cols), bool)
    for r, k in at:
        touched[r, k] = True
    if gated:
        touched[9, 3] = touched[11, cols - 1] = True
    same(a[~touched], a0[~touched])
    assert np.isinf(a[2, 5]) and np.isnan(a[4, 100]) and np.isnan(a[6, cols - 1])
    assert np.isnan(q[touched]).all() and not np.isnan(q[~touched]).any()
    with np.errstate(invalid="ignore"):
        wq, ws = ref.pack(np.where(touched, NAN, a), "row", "e4m3")
    if kind == "f32":            # (packed from the 32-bit values, which are a's bits here)
        same(q, wq)
        np.testing.assert_array_equal(s, ws)
    for k in range(many):
        wc, wsc = ref.pack(h[:, k * cols:(k + 1) * cols], "row", "e4m3")
        same(c[:, k * cols:(k + 1) * cols], wc)
        np.testing.assert_array_equal(sc[k * ref.blocks(cols):(k + 1) * ref.blocks(cols)], wsc)
    both = np.concatenate([touched] * many, 1)
    same(dh[~both], dh0[~both])
    assert np.isnan(dh[4, 100]) and np.isnan(dh[6, cols - 1]) and not np.isfinite(dh8[both]).all()


@pytest.mark.parametrize("to", ["e4m3", "e5m2"])
def test_repacking_values_that_are_not_finite(to):
    """Infinities and NaN of packed E5M2 values, and a scale byte 255, in every form of the new packing."""
    rows, cols = 140, 300
    rng = np.random.default_rng(4)
    q, s = ref.pack(data(rng, rows, cols), "row", "e5m2")
    q[3, 5], q[3, 200], q[131, 7], q[9, 290] = INF, -INF, NAN, INF
    s[0, 20] = 255
    x = q * ref.spread(ref.value_of(s), "row", rows, cols)
    t, ts = packed_up(q, s, "e5m2")
    d = mx.Quant8Desc.make(rows, cols, x_type=mx.DTYPE_E5M2, q_type=PACKED[to][0], ldx=t.stride(0))
    out = {f: (mx.empty_packed(rows, cols, PACKED[to][0]), mx.empty_scales(FORM[f], rows, cols)) for f in FORM}
    mx.quant8(d, t, x_scale=ts, **out)
    for f in FORM:
        want, ws = ref.pack(x, f, to)
        same(down(out[f][0]), want)
        np.testing.assert_array_equal(bytes_of(out[f][1]), ws)
