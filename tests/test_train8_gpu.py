"""The 8-bit training operators against their definitions in 64 bits.

Tolerances.  Packing multiplies by powers of two and rounds once: values and scales are
compared for equality.  A product sums on the tensor core (an error of at most one unit in the last place,
2^-23, of the running sum per MMA of 32 terms, at most 64 MMAs to an accumulator of an fp32 result and
4 per block of a 16-bit one, here of at most 14 blocks) and adds accumulators or blocks with one rounding each:
at most (128 + blocks) 2^-23 of sum |a b|.  Row sums of the layer norm
pass at most 64 additions from a value to the total: 64 x 2^-24 = 2^-18 of the sum of
magnitudes.  The activations' exponentials, error function and quotient are within a few units in the last
place: 2^-20 of the magnitudes that enter.  A result of 16 bits is compared with the rounded ends of its
interval."""
import numpy as np
import pytest
import torch

import paper_1501_06633_b200 as mx
import train8_ref as ref

pytestmark = pytest.mark.gpu

WIDE = {"f32": (mx.DTYPE_F32, torch.float32), "bf16": (mx.DTYPE_BF16, torch.bfloat16), "f16": (mx.DTYPE_F16, torch.float16)}
PACKED = {"e4m3": (mx.DTYPE_E4M3, torch.float8_e4m3fn), "e5m2": (mx.DTYPE_E5M2, torch.float8_e5m2)}
FORM = {"row": mx.BLOCK_ROW, "col": mx.BLOCK_COL, "tile": mx.BLOCK_TILE}
ACTS = {"silu": mx.ACT_SILU, "gelu": mx.ACT_GELU, "gelu_tanh": mx.ACT_GELU_TANH}


def up(a, dtype, ld=None):
    """A CUDA matrix with row pitch ld (its gaps hold NaN, which nothing may read)."""
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float64))
    if ld is None:
        return t.to(dtype).cuda()
    wide = torch.full((t.shape[0], ld), float("nan"), dtype=torch.float32).to(dtype).cuda()
    wide[:, :t.shape[1]] = t.to(dtype).cuda()
    return wide[:, :t.shape[1]]


def down(t):
    return t.to(torch.float32).double().cpu().numpy() if t.dtype != torch.float64 else t.cpu().numpy()


def packed_up(q, s, kind):
    """A packed operand from values and scale bytes (pitch: the next multiple of 16; its gaps hold
    NaN, which nothing may read)."""
    wide = torch.full((q.shape[0], -(-q.shape[1] // 16) * 16), 0x7F, dtype=torch.uint8, device="cuda")
    t = wide.view(PACKED[kind][1])[:, :q.shape[1]]
    bits = torch.from_numpy(q.astype(np.float32)).to(PACKED[kind][1]).view(torch.uint8)
    t.view(torch.uint8)[:] = bits.cuda()
    return t, torch.from_numpy(s).cuda().view(torch.float8_e8m0fnu)


def bytes_of(s):
    return s.view(torch.uint8).cpu().numpy()


def same(got, want):
    np.testing.assert_array_equal(np.isnan(got), np.isnan(want))
    np.testing.assert_array_equal(np.nan_to_num(got, nan=0.0, posinf=1e30, neginf=-1e30),
                                  np.nan_to_num(want, nan=0.0, posinf=1e30, neginf=-1e30))


def data(rng, rows, cols, spreading=True):
    x = rng.standard_normal((rows, cols))
    if spreading:
        x *= np.exp(2 * rng.standard_normal((rows, 1))) * np.exp(rng.standard_normal((1, cols)))
    return x


def as_held(x, kind):
    return down(torch.from_numpy(x).to(WIDE[kind][1]))


def within(got, want, tol, kind):
    """`got` is a value of [want - tol, want + tol] rounded to the type: rounding keeps order, so it
    lies between the ends' roundings."""
    with np.errstate(over="ignore"):
        assert np.all(got >= as_held(want - tol, kind)) and np.all(got <= as_held(want + tol, kind))


# ------------------------------------------------------------------ packing
@pytest.mark.parametrize("rows,cols,ldx", [(1, 1, None), (1, 128, None), (3, 130, None), (129, 127, None),
                                           (128, 128, 136), (257, 384, None), (40, 1000, 1003), (300, 17, 32)])
@pytest.mark.parametrize("xt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("qt", ["e4m3", "e5m2"])
def test_pack_every_form_at_once(rows, cols, ldx, xt, qt):
    rng = np.random.default_rng(rows * 1000 + cols)
    x = data(rng, rows, cols)
    x[0, 0] = 0.0
    if rows > 2:
        x[1] = 0.0
    x = as_held(x, xt)
    t = up(x, WIDE[xt][1], ldx)
    d = mx.Quant8Desc.make(rows, cols, x_type=WIDE[xt][0], q_type=PACKED[qt][0], ldx=ldx)
    out = {f: (mx.empty_packed(rows, cols, PACKED[qt][0]), mx.empty_scales(FORM[f], rows, cols)) for f in FORM}
    n0 = mx.launch_count()
    mx.quant8(d, t, **out)
    assert mx.launch_count() == n0 + 1
    for f in FORM:
        q, s = ref.pack(x, f, qt)
        same(down(out[f][0]), q)
        np.testing.assert_array_equal(bytes_of(out[f][1]), s)
        alone = (mx.empty_packed(rows, cols, PACKED[qt][0]), mx.empty_scales(FORM[f], rows, cols))
        mx.quant8(d, t, **{f: alone})
        same(down(alone[0]), q)
        np.testing.assert_array_equal(bytes_of(alone[1]), s)


@pytest.mark.parametrize("qt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("xt", ["f32", "bf16", "f16"])
def test_pack_extremes(xt, qt):
    """Largest and smallest magnitudes, the values around a change of the scale, infinities and NaN."""
    rows, cols = 130, 260
    rng = np.random.default_rng(5)
    x = data(rng, rows, cols, spreading=False)
    top = ref.SPEC[qt][0]
    big = {"f32": 3.0e38, "bf16": 3.0e38, "f16": 65504.0}[xt]
    x[0, 0], x[1, 130], x[2, 5] = big, -big, top
    x[3, :128] *= 0.001
    x[3, 7] = np.nextafter(np.float32(top), np.float32(np.inf)) if xt == "f32" else top * (1 + 2.0 ** -7)
    x[4] *= 1e-40 if xt != "f16" else 1e-7
    x[5] = 0.0
    x[6, 3], x[6, 140], x[7, 9] = np.inf, -np.inf, np.nan
    x[8, :] = np.inf
    x[9, :] = np.nan
    x[10] = 0.0
    x[10, 4] = 1e-45 if xt != "f16" else 6e-8
    with np.errstate(over="ignore"):
        x = as_held(x, xt)
    d = mx.Quant8Desc.make(rows, cols, x_type=WIDE[xt][0], q_type=PACKED[qt][0])
    out = {f: (mx.empty_packed(rows, cols, PACKED[qt][0]), mx.empty_scales(FORM[f], rows, cols)) for f in FORM}
    mx.quant8(d, up(x, WIDE[xt][1]), **out)
    for f in FORM:
        q, s = ref.pack(x, f, qt)
        np.testing.assert_array_equal(bytes_of(out[f][1]), s)
        same(down(out[f][0]), q)


@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 128), (131, 259), (256, 272)])
@pytest.mark.parametrize("kind", ["e4m3", "e5m2"])
def test_repack_and_unpack(rows, cols, kind):
    rng = np.random.default_rng(rows + cols)
    q, s = ref.pack(data(rng, rows, cols), "row", kind)
    x = q * ref.spread(ref.value_of(s), "row", rows, cols)
    t, ts = packed_up(q, s, kind)
    for to in PACKED:
        d = mx.Quant8Desc.make(rows, cols, x_type=PACKED[kind][0], q_type=PACKED[to][0], ldx=t.stride(0) if rows > 1 else None)
        if rows == 1:
            d.ldx = cols
        out = {f: (mx.empty_packed(rows, cols, PACKED[to][0]), mx.empty_scales(FORM[f], rows, cols)) for f in FORM}
        mx.quant8(d, t, x_scale=ts, **out)
        for f in FORM:
            want, ws = ref.pack(x, f, to)
            same(down(out[f][0]), want)
            np.testing.assert_array_equal(bytes_of(out[f][1]), ws)
    for f in FORM:
        qf, sf = ref.pack(x, f, kind)
        back = qf * ref.spread(ref.value_of(sf), f, rows, cols)
        tf, tsf = packed_up(qf, sf, kind)
        for xt, ldx in (("f32", cols), ("bf16", cols + 3), ("f16", cols + (-cols % 8))):
            wide = torch.full((rows, ldx), 7.0, dtype=WIDE[xt][1], device="cuda")
            d = mx.Quant8Desc.make(rows, cols, x_type=WIDE[xt][0], q_type=PACKED[kind][0], ldx=ldx)
            mx.dequant8(d, tf, tsf, wide[:, :cols], FORM[f])
            with np.errstate(over="ignore"):
                same(down(wide[:, :cols]), as_held(back, xt))
            assert bool((wide[:, cols:] == 7.0).all())


# ----------------------------------------------------------- matrix product
def gemm_case(rng, M, N, K, a_major, b_major, a_form, b_form, at, bt, zero_row=True):
    """Operands as stored, and the 64-bit result with the sum of magnitudes."""
    side = []
    for mn, major, form, kind in ((M, a_major, a_form, at), (N, b_major, b_form, bt)):
        x = data(rng, mn, K)
        if zero_row and mn > 1:
            x[mn // 2] = 0.0
        x = x if major == mx.MAJOR_K else np.ascontiguousarray(x.T)
        q, s = ref.pack(x, form, kind)
        v = q * ref.spread(ref.value_of(s), form, *x.shape)
        side.append((q, s, v if major == mx.MAJOR_K else v.T))
    return side[0], side[1], side[0][2] @ side[1][2].T, np.abs(side[0][2]) @ np.abs(side[1][2]).T


def check_gemm(got, want, mags, K, ct):
    within(got, want, (128 + ref.blocks(K)) * 2.0 ** -23 * mags, ct)


def run_gemm(M, N, K, a_major, b_major, a_form, b_form, at="e4m3", bt="e4m3", ct="f32", ldc=None, seed=0, f32_scales=""):
    rng = np.random.default_rng(seed)
    (qa, sa, _), (qb, sb, _), want, mags = gemm_case(rng, M, N, K, a_major, b_major, a_form, b_form, at, bt)
    ta, tsa = packed_up(qa, sa, at)
    tb, tsb = packed_up(qb, sb, bt)
    kinds = {}
    if "a" in f32_scales:
        tsa, kinds["a_scale_type"] = torch.from_numpy(ref.value_of(sa)).float().cuda(), mx.DTYPE_F32
    if "b" in f32_scales:
        tsb, kinds["b_scale_type"] = torch.from_numpy(ref.value_of(sb)).float().cuda(), mx.DTYPE_F32
    ldc = ldc or N
    wide = torch.full((M, ldc), 7.0, dtype=WIDE[ct][1], device="cuda")
    d = mx.Gemm8Desc.make(M, N, K, a_type=PACKED[at][0], b_type=PACKED[bt][0], c_type=WIDE[ct][0], a_major=a_major,
                          b_major=b_major, a_block=FORM[a_form], b_block=FORM[b_form], ldc=ldc, **kinds)
    mx.gemm8(d, ta, tsa, tb, tsb, wide[:, :N])
    assert mx.last_device_status() == mx.OK
    check_gemm(down(wide[:, :N]), want, mags, K, ct)
    assert bool((wide[:, N:] == 7.0).all())
    again = torch.empty_like(wide)
    mx.gemm8(d, ta, tsa, tb, tsb, again[:, :N])
    assert torch.equal(again[:, :N], wide[:, :N])


K_, MN_ = mx.MAJOR_K, mx.MAJOR_MN
WAYS = {"fprop": (K_, K_, "row", "tile"), "dgrad": (K_, MN_, "row", "tile"), "wgrad": (MN_, MN_, "col", "col"),
        "both rows": (K_, K_, "row", "row"), "tiles": (MN_, K_, "tile", "tile")}


@pytest.mark.parametrize("way", list(WAYS))
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 256, 128), (7, 130, 129), (128, 128, 128), (129, 257, 300),
                                   (200, 96, 1000), (300, 520, 77), (64, 1000, 640)])
def test_gemm_sizes_and_majors(way, M, N, K):
    run_gemm(M, N, K, *WAYS[way], seed=M + N + K)


@pytest.mark.parametrize("cols", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("split", [1, 2, 8])
@pytest.mark.parametrize("swap", [0, 1])
@pytest.mark.parametrize("way", ["fprop", "wgrad"])
def test_gemm_every_plan_with_fp32_scales(cols, split, swap, way):
    mx.set_option("GEMM8_COLS", cols)
    mx.set_option("GEMM8_SPLIT", split)
    mx.set_option("GEMM8_SWAP", swap)
    run_gemm(150, 330, 1100, *WAYS[way], ct="bf16", seed=cols + split, f32_scales="ab")


@pytest.mark.parametrize("pair,cols,split", [(-1, c, s) for c in (16, 32, 64, 128) for s in (1, 2, 4, 8)] +
                         [(1, c, 1) for c in (128, 192, 224, 256)])
@pytest.mark.parametrize("swap", [0, 1])
@pytest.mark.parametrize("way", ["fprop", "dgrad", "wgrad"])
@pytest.mark.parametrize("ct,ldc", [("bf16", 336), ("f32", 336), ("f16", 331)])
def test_gemm_every_plan(pair, cols, split, swap, way, ct, ldc):
    mx.set_option("GEMM8_PAIR", pair)
    mx.set_option("GEMM8_COLS", cols)
    mx.set_option("GEMM8_SPLIT", split)
    mx.set_option("GEMM8_SWAP", swap)
    run_gemm(150, 330, 1100, *WAYS[way], ct=ct, ldc=ldc, seed=cols + split)


@pytest.mark.parametrize("pair,cols", [(-1, 128), (1, 128), (1, 192), (1, 224), (1, 256)])
def test_gemm_many_tiles_and_chunks(pair, cols):
    """More tiles than SMs, several accumulator chunks: every buffer and barrier goes around."""
    mx.set_option("GEMM8_PAIR", pair)
    mx.set_option("GEMM8_COLS", cols)
    run_gemm(2300, 5000, 1700, *WAYS["fprop"], seed=cols)
    run_gemm(2300, 5000, 700, *WAYS["wgrad"], ct="bf16", seed=cols)


@pytest.mark.parametrize("at,bt", [("e4m3", "e5m2"), ("e5m2", "e4m3"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("ct,ldc", [("f32", None), ("bf16", 336), ("f16", 331)])
@pytest.mark.parametrize("way", ["fprop", "dgrad", "wgrad"])
def test_gemm_types_and_pitches(at, bt, ct, ldc, way):
    run_gemm(140, 330, 260, *WAYS[way], at=at, bt=bt, ct=ct, ldc=ldc, seed=3)


@pytest.mark.parametrize("which", ["a", "b", "ab"])
@pytest.mark.parametrize("way", ["fprop", "wgrad"])
def test_gemm_fp32_scales(which, way):
    run_gemm(140, 270, 390, *WAYS[way], f32_scales=which, seed=4)


def test_gemm_arbitrary_fp32_scales_and_special_values():
    """Scales that are no powers of two; NaN and infinity reach their row and column and no other."""
    M, N, K = 130, 200, 256
    rng = np.random.default_rng(8)
    qa, _ = ref.pack(data(rng, M, K, False), "row", "e5m2")
    qb, _ = ref.pack(data(rng, N, K, False), "tile", "e4m3")
    fa, fb = rng.uniform(0.3, 3.0, (2, M)).astype(np.float32), rng.uniform(0.3, 3.0, (2, 2)).astype(np.float32)
    qa[5, 7], qb[9, 200] = np.inf, np.nan
    qb[:, 7] = np.where(qb[:, 7] == 0, 1.0, qb[:, 7])
    ta, _ = packed_up(qa, np.zeros((2, M), np.uint8), "e5m2")
    tb, _ = packed_up(qb, np.zeros((2, 2), np.uint8), "e4m3")
    c = torch.empty(M, N, device="cuda")
    d = mx.Gemm8Desc.make(M, N, K, a_type=mx.DTYPE_E5M2, c_type=mx.DTYPE_F32, a_scale_type=mx.DTYPE_F32, b_scale_type=mx.DTYPE_F32)
    mx.gemm8(d, ta, torch.from_numpy(fa).cuda(), tb, torch.from_numpy(fb).cuda(), c)
    got = down(c)
    va = qa * ref.spread(fa.astype(np.float64), "row", M, K)
    vb = qb * ref.spread(fb.astype(np.float64), "tile", N, K)
    clean_a, clean_b = np.where(np.isfinite(va), va, 0), np.where(np.isfinite(vb), vb, 0)
    want, mags = clean_a @ clean_b.T, np.abs(clean_a) @ np.abs(clean_b).T
    touched = np.zeros((M, N), bool)
    touched[5], touched[:, 9] = True, True
    assert np.isnan(got[:, 9]).all()
    others = np.delete(np.arange(N), 9)
    assert not np.isfinite(got[5, others]).any()
    tol = (128 + 2 + 2) * 2.0 ** -23 * mags
    assert np.all(np.abs(got - want)[~touched] <= tol[~touched])


def test_gemm_long_reduction_of_equal_signs():
    """32768 terms of one sign: the blocks' sums keep the error at a block's, not the length's."""
    M, N, K = 128, 128, 32768
    qa, sa = ref.pack(np.full((M, K), 1.0625), "row", "e4m3")
    qb, sb = ref.pack(np.full((N, K), 0.9375), "tile", "e4m3")
    va = qa * ref.spread(ref.value_of(sa), "row", M, K)
    vb = qb * ref.spread(ref.value_of(sb), "tile", N, K)
    (ta, tsa), (tb, tsb) = packed_up(qa, sa, "e4m3"), packed_up(qb, sb, "e4m3")
    c = torch.empty(M, N, device="cuda")
    mx.gemm8(mx.Gemm8Desc.make(M, N, K, c_type=mx.DTYPE_F32), ta, tsa, tb, tsb, c)
    want = va @ vb.T
    # sums of 256 blocks in fp32: at most one rounding of 2^-24 each
    assert np.max(np.abs(down(c) - want) / want) <= 256 * 2.0 ** -24


def test_gemm_empty_sizes():
    c = torch.full((5, 9), 3.0, device="cuda")
    d = mx.Gemm8Desc.make(5, 9, 0, c_type=mx.DTYPE_F32, lda=16, ldb=16)
    e8 = lambda *s: torch.empty(*s, dtype=torch.uint8, device="cuda")
    mx.gemm8(d, e8(5, 0), e8(0, 5), e8(9, 0), e8(1, 0), c)
    assert bool((c == 0).all())
    n0 = mx.launch_count()
    d = mx.Gemm8Desc.make(0, 9, 32, c_type=mx.DTYPE_F32)
    mx.gemm8(d, e8(0, 32), e8(1, 0), e8(9, 32), e8(1, 1), torch.empty(0, 9, device="cuda"))
    assert mx.launch_count() == n0


# --------------------------------------------------------------- layer norm
SUM_TOL = 2.0 ** -18


def near_packed(q, s, x, tol, kind):
    """q, s hold x: within half a step of the 8-bit type, and tol."""
    top, bits, least, _ = ref.SPEC[kind]
    scale = ref.spread(ref.value_of(bytes_of(s)), "row", *x.shape)
    v = down(q) * scale
    m = np.maximum(np.abs(x), 2.0 ** least * scale)
    half = 2.0 ** (np.floor(np.log2(m)) - bits - 1)
    assert np.all(np.abs(v - x) <= half * 1.0001 + tol)
    for at, rs, cs in ref.cells("row", *x.shape):
        peak, slack = np.max(np.abs(x[rs, cs])), np.max(tol[rs, cs])
        sc = ref.value_of(bytes_of(s))[at]
        if peak > slack:
            assert top * sc >= peak - slack and (top * sc / 2 <= peak + slack or sc == 2.0 ** -126)


@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (2, 7, 0), (5, 64, 0), (3, 1000, 0), (9, 1024, 8), (4, 1025, 3), (6, 2048, 0),
                                           (3, 4096, 0), (2, 4100, 0), (3, 8192, 0), (2, 9000, 0), (2, 16384, 0),
                                           (2, 16392, 0), (2, 20001, 0)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_layer_norm_fprop(rows, cols, pad, kind):
    rng = np.random.default_rng(cols)
    x = as_held(3.0 * data(rng, rows, cols, False) + 5.0, kind)
    gamma, beta = rng.uniform(-2, 2, cols), rng.standard_normal(cols)
    wk = "f32" if kind == "f32" else kind
    gamma, beta = as_held(gamma, wk), as_held(beta, wk)
    want, mean, rstd = ref.layer_norm(x, gamma, beta, 1e-5)
    code, tt = WIDE[kind]
    d = mx.LayerNormDesc.make(rows, cols, x_type=code, w_type=WIDE[wk][0], ldx=cols + pad, ldy=cols + pad)
    t = up(x, tt, cols + pad)
    y = torch.full((rows, cols + pad), 7.0, dtype=tt, device="cuda")
    m, r = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    q, c = mx.empty_packed(rows, cols), mx.empty_packed(rows, cols)
    s, sc = mx.empty_scales(mx.BLOCK_ROW, rows, cols), mx.empty_scales(mx.BLOCK_ROW, rows, cols)
    g, b = up(gamma, WIDE[wk][1]), up(beta, WIDE[wk][1])
    mx.layer_norm_fprop(d, t, g, b, y=y[:, :cols], mean=m, rstd=r, packed=(q, s), checkpoint=(c, sc))
    size = np.abs(x).mean(1)
    assert np.all(np.abs(down(m) - mean) <= SUM_TOL * size)
    # the mean's error enters the differences; the variance is relative to itself (eps where it vanishes)
    rel = 2 * SUM_TOL + 4 * SUM_TOL * size * rstd
    assert np.all(np.abs(down(r) - rstd) <= rel * rstd)
    tol = (rel[:, None] + 2.0 ** -22) * (np.abs((want - beta)) + np.abs(gamma)) + 2.0 ** -22 * np.abs(want)
    within(down(y[:, :cols]), want, tol, kind)
    assert bool((y[:, cols:] == 7.0).all())
    near_packed(q, s, want, tol, "e4m3")
    wq, ws = ref.pack(x, "row", "e4m3")
    same(down(c), wq)
    np.testing.assert_array_equal(bytes_of(sc), ws)
    # any result alone, and no weights
    only = torch.empty(rows, cols, dtype=tt, device="cuda")
    d2 = mx.LayerNormDesc.make(rows, cols, x_type=code, ldx=cols + pad)
    mx.layer_norm_fprop(d2, t, y=only)
    plain, _, _ = ref.layer_norm(x, 1.0, 0.0, 1e-5)
    within(down(only), plain, (rel[:, None] + 2.0 ** -22) * (np.abs(plain) + 1), kind)


def test_layer_norm_far_from_zero_and_constant_rows():
    """Rows at 1000 with a spread of 1, one huge column, and a row of equal values (variance 0)."""
    rows, cols = 4, 3000
    rng = np.random.default_rng(2)
    x = np.float32(1000 + rng.standard_normal((rows, cols))).astype(np.float64)
    x[1, 17] = 1e6
    x[2] = 42.0
    want, mean, rstd = ref.layer_norm(x, 1.0, 0.0, 1e-5)
    y, r = torch.empty(rows, cols, device="cuda"), torch.empty(rows, device="cuda")
    mx.layer_norm_fprop(mx.LayerNormDesc.make(rows, cols, x_type=mx.DTYPE_F32), up(x, torch.float32), y=y, rstd=r)
    size = np.abs(x).mean(1)
    rel = 2 * SUM_TOL + 4 * SUM_TOL * size * np.where(np.arange(rows) == 2, 0.0, rstd)
    assert np.all(np.abs(down(r) - rstd) <= rel * rstd)
    assert np.all(np.abs(down(y) - want) <= rel[:, None] * (np.abs(want) + 1) + 2.0 ** -22)


@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 7, 0), (70, 64, 0), (601, 300, 0), (33, 1024, 8), (20, 1025, 3),
                                           (700, 2048, 0), (5, 4100, 0), (9, 8192, 0), (3, 8200, 0), (4, 20001, 0)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("packed", [None, "e4m3", "e5m2"])
def test_layer_norm_bprop(rows, cols, pad, kind, packed):
    rng = np.random.default_rng(rows + cols)
    x = as_held(2.0 * data(rng, rows, cols, False) + 1.0, kind)
    dy, gamma = as_held(data(rng, rows, cols, False), kind), rng.uniform(-2, 2, cols).astype(np.float32).astype(np.float64)
    _, mean, rstd = ref.layer_norm(x, 1.0, 0.0, 1e-5)
    mean, rstd = np.float32(mean).astype(np.float64), np.float32(rstd).astype(np.float64)
    code, tt = WIDE[kind]
    if packed:
        q, s = ref.pack(x, "row", packed)
        x = q * ref.spread(ref.value_of(s), "row", rows, cols)
        t, ts = packed_up(q, s, packed)
        d = mx.LayerNormDesc.make(rows, cols, x_type=PACKED[packed][0], y_type=code, ldx=t.stride(0), ldy=cols + pad)
    else:
        t, ts = up(x, tt, cols + pad), None
        d = mx.LayerNormDesc.make(rows, cols, x_type=code, ldx=cols + pad, ldy=cols + pad)
    dx = torch.full((rows, cols + pad), 7.0, dtype=tt, device="cuda")
    dg, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(mx.layer_norm_bprop_workspace(d), dtype=torch.uint8, device="cuda")
    g, m, r = (up(v, torch.float32) for v in (gamma, mean, rstd))
    mx.layer_norm_bprop(d, up(dy, tt, cols + pad), t, g, m, r, dx[:, :cols], dg, db, ws, x_scale=ts)
    want, wg, wb = ref.layer_norm_grads(x, dy, gamma, mean, rstd)
    xh = (x - mean[:, None]) * rstd[:, None]
    xh_err = 2.0 ** -22 * (np.abs(x) + np.abs(mean[:, None])) * rstd[:, None]
    e = np.abs(dy * gamma)
    s1, s2 = e.mean(1, keepdims=True), (e * np.abs(xh)).mean(1, keepdims=True)
    tol = rstd[:, None] * (SUM_TOL * (e + s1 + np.abs(xh) * s2) + xh_err * s2 + np.abs(xh) * (e * xh_err).mean(1, keepdims=True))
    within(down(dx[:, :cols]), want, tol, kind)
    assert bool((dx[:, cols:] == 7.0).all())
    # sums over rows: at most rows roundings, as one chain or several
    row_tol = (rows + 32) * 2.0 ** -24
    assert np.all(np.abs(down(dg) - wg) <= row_tol * np.abs(dy * xh).sum(0) + (np.abs(dy) * xh_err).sum(0) + 1e-30)
    assert np.all(np.abs(down(db) - wb) <= row_tol * np.abs(dy).sum(0) + 1e-30)
    # one of the sums alone, and neither
    one = torch.empty(cols, device="cuda")
    again = torch.empty_like(dx)
    mx.layer_norm_bprop(d, up(dy, tt, cols + pad), t, g, m, r, again[:, :cols], None, one, ws, x_scale=ts)
    assert torch.equal(one, db) and torch.equal(again[:, :cols], dx[:, :cols])
    again.fill_(7.0)
    mx.layer_norm_bprop(d, up(dy, tt, cols + pad), t, g, m, r, again[:, :cols], x_scale=ts)
    assert torch.equal(again, dx)


def test_layer_norm_gradients_against_differences():
    rows, cols, h = 3, 40, 1e-2
    rng = np.random.default_rng(0)
    x, dy = np.float32(data(rng, rows, cols, False)), np.float32(data(rng, rows, cols, False))
    gamma, beta = np.float32(rng.uniform(0.5, 1.5, cols)), np.float32(rng.standard_normal(cols))
    d = mx.LayerNormDesc.make(rows, cols, x_type=mx.DTYPE_F32)

    def loss(x, gamma, beta):
        y = torch.empty(rows, cols, device="cuda")
        mx.layer_norm_fprop(d, torch.from_numpy(x).cuda(), torch.from_numpy(gamma).cuda(), torch.from_numpy(beta).cuda(), y=y)
        return float((down(y) * dy).sum())

    m, r = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    tx, tg = torch.from_numpy(x).cuda(), torch.from_numpy(gamma).cuda()
    mx.layer_norm_fprop(d, tx, tg, mean=m, rstd=r)
    dx, dg, db = torch.empty(rows, cols, device="cuda"), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(mx.layer_norm_bprop_workspace(d), dtype=torch.uint8, device="cuda")
    mx.layer_norm_bprop(d, torch.from_numpy(dy).cuda(), tx, tg, m, r, dx, dg, db, ws)
    # central differences: h^2 times a third derivative of a few units, and the forward pass's
    # fp32 rounding (about 1e-6 of a sum of 120 terms) over 2 h
    tol = 50 * h * h * 0.1 + 1e-5 / (2 * h)
    for grad, of in ((down(dx), 0), (down(dg), 1), (down(db), 2)):
        for at in ((0, 0), (1, 17), (2, 39)) if of == 0 else ((0,), (17,), (39,)):
            args = [x.copy(), gamma.copy(), beta.copy()]
            args[of][at] += h
            high = loss(*args)
            args[of][at] -= 2 * h
            assert abs((high - loss(*args)) / (2 * h) - grad[at]) <= tol


# --------------------------------------------------------------- activation
ACT_TOL = 2.0 ** -20


@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 128, 0), (65, 130, 0), (64, 264, 8), (100, 77, 1), (7, 1000, 0)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("gated", [True, False])
def test_act8(rows, cols, pad, kind, act, gated):
    rng = np.random.default_rng(rows + cols)
    many = 2 if gated else 1
    code, tt = WIDE[kind]
    h = as_held(3.0 * data(rng, rows, many * cols, False), kind)
    h[0, 0] = 0.0
    if cols > 20:
        h[0, 1:5] = [-100.0, 100.0, -30.0, 12.0]
    g, u = h[:, :cols], h[:, cols:] if gated else 1.0
    f, df = ref.act(act, g)
    ldh, lda = many * cols + pad, cols + pad
    d = mx.Act8Desc.make(rows, cols, act=ACTS[act], gated=gated, x_type=code, ldh=ldh, lda=lda)
    th = up(h, tt, ldh)
    a = torch.full((rows, lda), 7.0, dtype=tt, device="cuda")
    q, s = mx.empty_packed(rows, cols), mx.empty_scales(mx.BLOCK_ROW, rows, cols)
    c = mx.empty_packed(rows, many * cols)
    sc = torch.empty(many * ref.blocks(cols), rows, dtype=torch.uint8, device="cuda")
    mx.act8_fprop(d, th, a=a[:, :cols], packed=(q, s), checkpoint=(c, sc))
    want = f * u
    tol = ACT_TOL * np.abs(g * u)
    within(down(a[:, :cols]), want, tol, kind)
    assert bool((a[:, cols:] == 7.0).all())
    near_packed(q, s, want, tol, "e4m3")
    parts = [ref.pack(h[:, k * cols:(k + 1) * cols], "row", "e4m3") for k in range(many)]
    same(down(c), np.concatenate([p[0] for p in parts], 1))
    np.testing.assert_array_equal(sc.cpu().numpy(), np.concatenate([p[1] for p in parts], 0))
    q2, s2 = mx.empty_packed(rows, cols), mx.empty_scales(mx.BLOCK_ROW, rows, cols)
    mx.act8_fprop(d, th, packed=(q2, s2))
    assert torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(s2.view(torch.uint8), s.view(torch.uint8))

    # backward, from h and from what was kept of it
    da = as_held(data(rng, rows, cols, False), kind)
    tda = up(da, tt, lda)
    kept = np.concatenate([p[0] * ref.spread(ref.value_of(p[1]), "row", rows, cols) for p in parts], 1)
    for packed in (False, True):
        hv = kept if packed else h
        gv, uv = hv[:, :cols], hv[:, cols:] if gated else 1.0
        fv, dfv = ref.act(act, gv)
        dh = torch.full((rows, ldh), 7.0, dtype=tt, device="cuda")
        db = mx.Act8Desc.make(rows, cols, act=ACTS[act], gated=gated, x_type=code, ldh=ldh, lda=lda,
                              h_type=mx.DTYPE_E4M3 if packed else None)
        mx.act8_bprop(db, tda, c if packed else th, dh[:, :many * cols], h_scale=sc if packed else None)
        got = down(dh[:, :many * cols])
        w = da * uv * dfv
        # far out, f' is a difference of terms as large as g
        t1 = ACT_TOL * np.abs(da * uv) * (1 + np.minimum(np.abs(gv), 20.0))
        within(got[:, :cols], w, t1, kind)
        if gated:
            w = da * fv
            within(got[:, cols:], w, ACT_TOL * np.abs(da * gv), kind)
        assert bool((dh[:, many * cols:] == 7.0).all())


@pytest.mark.parametrize("act", list(ACTS))
def test_act8_gradient_against_differences(act):
    rows, cols, step = 4, 64, 2.0 ** -7
    g = np.linspace(-4, 4, rows * cols).reshape(rows, cols).astype(np.float32)
    d = mx.Act8Desc.make(rows, cols, act=ACTS[act], gated=False, x_type=mx.DTYPE_F32)

    def f(x):
        a = torch.empty(rows, cols, device="cuda")
        mx.act8_fprop(d, torch.from_numpy(np.ascontiguousarray(x)).cuda(), a=a)
        return down(a)

    dh = torch.empty(rows, cols, device="cuda")
    mx.act8_bprop(d, torch.ones(rows, cols, device="cuda"), torch.from_numpy(g).cuda(), dh)
    numeric = (f(g + np.float32(step)) - f(g - np.float32(step))) / (2 * step)
    # step^2 / 6 times a third derivative below 3, and fp32 rounding of values up to 4 over 2 step
    assert np.max(np.abs(numeric - down(dh))) <= 0.5 * step * step + 4 * 2.0 ** -22 / step


# ------------------------------------------------------- streams and offsets
def test_other_stream_and_graph():
    """Every call on a stream of its own, captured and replayed with new data."""
    rows, cols, out = 96, 256, 384
    rng = np.random.default_rng(1)
    x = up(data(rng, rows, cols, False), torch.bfloat16)
    q, s = mx.empty_packed(rows, cols), mx.empty_scales(mx.BLOCK_ROW, rows, cols)
    w, ws = mx.empty_packed(out, cols), mx.empty_scales(mx.BLOCK_TILE, out, cols)
    y = torch.empty(rows, out, dtype=torch.bfloat16, device="cuda")
    mx.quant8(mx.Quant8Desc.make(out, cols), up(data(rng, out, cols, False), torch.bfloat16), tile=(w, ws))
    ln, gm = mx.LayerNormDesc.make(rows, cols), mx.Gemm8Desc.make(rows, out, cols)
    stream = torch.cuda.Stream()

    def both():
        mx.layer_norm_fprop(ln, x, packed=(q, s), stream=stream)
        mx.gemm8(gm, q, s, w, ws, y, stream=stream)

    stream.wait_stream(torch.cuda.current_stream())
    both()
    stream.synchronize()
    first = y.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        both()
    x.mul_(-1.0)
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, -first)
    assert mx.last_device_status() == mx.OK


def test_offsets_beyond_32_bits():
    """The last rows of a matrix of more than 2^32 bytes (and 2^31 elements)."""
    cols, rows = 4096, 600000
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    rng = np.random.default_rng(3)
    last = as_held(data(rng, 130, cols), "bf16")
    x[-130:] = up(last, torch.bfloat16)
    q, s = mx.empty_packed(rows, cols), mx.empty_scales(mx.BLOCK_ROW, rows, cols)
    mx.quant8(mx.Quant8Desc.make(rows, cols), x, row=(q, s))
    wq, wsc = ref.pack(last, "row", "e4m3")
    same(down(q[-130:]), wq)
    np.testing.assert_array_equal(bytes_of(s)[:, -130:], wsc)
    y = torch.empty_like(x)
    mx.layer_norm_fprop(mx.LayerNormDesc.make(rows, cols), x, y=y)
    want, _, _ = ref.layer_norm(last, 1.0, 0.0, 1e-5)
    size, rstd = np.abs(last).mean(1, keepdims=True), 1 / last.std(1, keepdims=True)
    within(down(y[-130:]), want, (2 * SUM_TOL + 4 * SUM_TOL * size * rstd + 2.0 ** -22) * (np.abs(want) + 1), "bf16")
    w, wt = ref.pack(data(rng, 64, cols, False), "tile", "e4m3")
    (tw, tws), c = packed_up(w, wt, "e4m3"), torch.empty(rows, 64, device="cuda")
    mx.gemm8(mx.Gemm8Desc.make(rows, 64, cols, c_type=mx.DTYPE_F32), q, s, tw, tws, c)
    va = wq * ref.spread(ref.value_of(wsc), "row", 130, cols)
    vb = w * ref.spread(ref.value_of(wt), "tile", 64, cols)
    check_gemm(down(c[-130:]), va @ vb.T, np.abs(va) @ np.abs(vb).T, cols, "f32")


def test_a_wait_that_runs_out_ends_in_a_status():
    d = mx.Gemm8Desc.make(128, 128, 256, c_type=mx.DTYPE_F32)
    e8 = lambda *s: torch.zeros(*s, dtype=torch.uint8, device="cuda")
    args = (e8(128, 256), e8(2, 128), e8(128, 256), e8(1, 2), torch.empty(128, 128, device="cuda"))
    mx.gemm8(d, *args)
    assert mx.last_device_status() == mx.OK
    mx.set_option("TEST_MISSING_ARRIVAL", 1)
    mx.gemm8(d, *args)
    assert mx.last_device_status() == mx.DEVICE_TIMEOUT
    mx.unset_option("TEST_MISSING_ARRIVAL")
    mx.gemm8(d, *args)
    assert mx.last_device_status() == mx.OK
