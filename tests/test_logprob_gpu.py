"""Log probabilities, entropy, alternatives and their gradient against their definitions in 64 bits.

Tolerances, with A and A2 the mean and mean square distance to the row's maximum under p.  A difference to the maximum
in powers of two has four roundings (2^-22 of itself, the factor's two among them), the exponential 2^-22: a term's relative error is
2^-22 (1 + distance).  Sums pass at most 128 additions and rescalings: 2^-17.  So ln S is within 2^-17 + 2^-22 A, and the
entropy within 2^-17 (1 + A) + 2^-22 (A + A2) more.  Gradients: see logprob_ref.py; ln p has one rounding, its multiple of
log2 e two, p 2^-22 more, the factor behind it four."""
import numpy as np
import pytest
import torch

import logprob_ref as ref
import paper_1501_06633_b200 as mx
from packed_rows import near_rows
from test_train8_gpu import PACKED, WIDE, as_held, down, up, within

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def logits(rng, rows, cols, kind):
    x = 3 * rng.standard_normal((rows, cols)) + 10 * (rng.random((rows, cols)) < 4 / cols)
    x[:, rng.random(cols) < 0.05] = -np.inf
    return as_held(x, kind)


def close(got, want, tol):
    fine = np.isfinite(want)
    np.testing.assert_array_equal(got[~fine], want[~fine])
    assert np.all(np.abs(got[fine] - want[fine]) <= np.broadcast_to(tol, want.shape)[fine])


def forward(x, kind, scale=1.0, target=None, top=0, ld=None, wide=True):
    rows, cols = x.shape
    code, tt = WIDE[kind]
    d = mx.LogprobDesc.make(rows, cols, top=top, scale=scale, x_type=code, ldx=ld, target_type=mx.INDEX_I64 if wide else mx.INDEX_I32)
    new = lambda *s: torch.full(s, 99.0, device="cuda")
    out = {"lse": new(rows), "entropy": new(rows)}
    if target is not None:
        out["logprob"] = new(rows)
        target = torch.from_numpy(target).to(torch.int64 if wide else torch.int32).cuda()
    if top:
        out.update(top_logprob=new(rows, top), top_index=torch.full((rows, top), -7, dtype=torch.int32, device="cuda"))
    mx.logprob_fprop(d, up(x, tt, ld), target, **out)
    assert mx.last_device_status() == mx.OK
    return {k: v.cpu().numpy().astype(np.float64) for k, v in out.items()}


def check(x, kind, scale, target, top, ld=None, wide=True):
    got = forward(x, kind, scale, target, top, ld, wide)
    lse, lp, entropy, tlp, idx, a1, a2 = ref.forward(x, scale, target, max(top, 1))
    ln = 2.0 ** -17 + 2.0 ** -22 * a1
    with np.errstate(invalid="ignore"):
        m = np.where(np.isfinite(x).any(1), np.max(np.where(np.isfinite(x), x, -np.inf), 1), 0.0) * scale
    tol = ln + 4 * U * (np.abs(m) + np.abs(np.where(np.isfinite(lse), lse, 0)))
    close(got["lse"], lse, tol)
    close(got["logprob"], lp, ln + 4 * U * np.abs(np.where(np.isfinite(lp), lp, 0)) + 4 * U * np.abs(m) * (scale != 1))
    close(got["entropy"], entropy, ln + 2.0 ** -17 * (1 + a1) + 2.0 ** -22 * (a1 + a2))
    if top:
        np.testing.assert_array_equal(got["top_index"], idx)
        close(got["top_logprob"], tlp, ln[:, None] + 4 * U * np.abs(np.where(np.isfinite(tlp), tlp, 0)))


# columns: shorter than a vector, odd, a thread's single values on both ends, rows shared by 2, 4 and 8 CTAs and by one
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (2, 3, 0), (3, 7, 1), (5, 100, 0), (4, 257, 0), (3, 2049, 0), (7, 4097, 3), (1, 8191, 0),
                                           (3, 8192, 0), (2, 20001, 7), (1, 65537, 0), (80, 16411, 0), (250, 8200, 0), (640, 1003, 0)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_forward(rows, cols, pad, kind):
    rng = np.random.default_rng(rows * 7 + cols)
    x = logits(rng, rows, cols, kind)
    target = rng.integers(0, cols, rows)
    target[::3] = -100
    target[1::5] = cols
    for top, scale, wide in ((0, 1.0, True), (1, 1.0, False), (5, 0.75, True), (32, 1.0, False)):
        check(x, kind, scale, target, top, cols + pad, wide)
    # one result alone is the same
    full = forward(x, kind, 1.0, target, 5)
    d = mx.LogprobDesc.make(rows, cols, x_type=WIDE[kind][0])
    lp = torch.empty(rows, device="cuda")
    mx.logprob_fprop(d, up(x, WIDE[kind][1]), torch.from_numpy(target).cuda(), logprob=lp)
    np.testing.assert_array_equal(down(lp), full["logprob"])


@pytest.mark.parametrize("rows,cols", [(1, 20000), (2, 40003), (600, 5000)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_alternatives_where_values_are_equal_or_masked(rows, cols, kind):
    """Rows of one value; masks by the type's lowest value and by -inf that leave one, a few or no token; rising and falling
    rows; few different values; the large values at one place of each thread's stride; zeros of both signs."""
    code, tt = WIDE[kind]
    rng = np.random.default_rng(3)
    lowest = float(torch.finfo(tt).min)
    n = np.arange(cols)
    patterns = [np.zeros(cols), np.full(cols, lowest), np.full(cols, -np.inf), np.where(n == cols // 2, 1.0, lowest),
                np.where(np.isin(n, (5, 700, cols - 1)), [1.0], lowest), np.where(np.isin(n, (5, 700, cols - 1)), 2.0, -np.inf),
                np.where(n == cols - 1, -3.0, -np.inf), n * (100.0 / cols), -n * (100.0 / cols), rng.integers(0, 3, cols).astype(float),
                np.where(n % 2048 == 17, 50 + n / cols, rng.standard_normal(cols)), np.where(n % 2048 < 8, 50.0, 0.0),
                np.where(n % 2, 0.0, -0.0), np.where(n % (256 * 4) < 4, n * 1e-3, -5.0)]
    for i, row in enumerate(patterns):
        x = logits(rng, rows, cols, kind)
        x[0] = x[-1] = as_held(row[None], kind)[0]
        target = rng.integers(0, cols, rows)
        target[0] = (5, -1)[i % 2]
        check(x, kind, 1.0, target, 32)
        check(x, kind, 1.0, target, 3)


@pytest.mark.parametrize("rows,cols,pad", [(1, 131072, 0), (2, 150001, 7), (20, 131079, 0), (60, 65539, 5), (76, 131100, 0), (140, 33000, 0)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_long_rows_that_ctas_share(rows, cols, pad, kind):
    """By 8, 8, 8, 4, 2 and 2 CTAs; rows with one token, with none, of one value, and with their tokens in one CTA's part."""
    rng = np.random.default_rng(cols)
    x = logits(rng, rows, cols, kind)
    target = rng.integers(0, cols, rows)
    target[1::5] = -1
    n = np.arange(cols)
    special = [np.where(n == cols - 1, 2.0, -np.inf), np.full(cols, -np.inf), np.full(cols, 3.0), np.where(n < 40, n * 0.25, -np.inf),
               np.where(n >= cols - 9, n - cols, float(torch.finfo(WIDE[kind][1]).min))]
    check(x, kind, 0.75, target, 32, cols + pad)
    for i, row in enumerate(special):
        if rows > 2 and i < len(special) - 1:      # all at once
            x[(i + 1) * rows // 6] = as_held(row[None], kind)[0]
            continue
        x[0] = as_held(row[None], kind)[0]
        target[0] = (cols - 1, 3)[i % 2]
        check(x, kind, 1.0, target, 20, cols + pad, i % 2 == 0)


@pytest.mark.parametrize("rows,threads", [(300, 256), (900, 128)])
def test_alternatives_of_long_rows_whose_large_values_lie_close_together(rows, threads):
    """More values above the bound than there is room for, in fewer threads than alternatives: the rows' large values lie at one
    place of the threads' stride; in others all values but a few are equal."""
    cols = 150000
    gen = torch.Generator(device="cuda").manual_seed(8)
    x = torch.randn(rows, cols, device="cuda", generator=gen).to(torch.bfloat16)
    n = np.arange(cols)
    rng = np.random.default_rng(4)
    special = {0: np.where((n // 8) % threads < 4, 20 + 10 * rng.random(cols), -rng.random(cols)),
               7: np.where((n // 8) % threads < 8, 20 + n * 1e-4, 0.0), rows - 1: np.where(n % 50021 == 3, 5.0, -7.0)}
    for r, v in special.items():
        x[r] = torch.from_numpy(as_held(v[None], "bf16")[0]).to(torch.bfloat16).cuda()
    for top in (3, 32):
        v, at = torch.empty(rows, top, device="cuda"), torch.empty(rows, top, dtype=torch.int32, device="cuda")
        lse = torch.empty(rows, device="cuda")
        mx.logprob_fprop(mx.LogprobDesc.make(rows, cols, top=top), x, lse=lse, top_logprob=v, top_index=at)
        some = [*special, 1, rows // 2]
        want, _, _, tlp, idx, a1, _ = ref.forward(down(x[some]), 1.0, np.full(len(some), -1), top)
        np.testing.assert_array_equal(at[some].cpu().numpy(), idx)
        close(down(v[some]), tlp, (2.0 ** -17 + 2.0 ** -22 * a1)[:, None] + 4 * U * np.abs(tlp))


@pytest.mark.parametrize("cols", [300, 9000, 70000])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_rows_that_are_not_finite(cols, kind):
    rng = np.random.default_rng(5)
    x = logits(rng, 6, cols, kind)
    x[1, 7], x[2, cols - 1], x[3, 0], x[4] = np.nan, np.inf, np.nan, -np.inf
    x[4, 9] = np.nan
    target = np.array([1, 2, 3, -1, 4, 5])
    got = forward(x, kind, 1.0, target, 4)
    for name in ("lse", "entropy"):
        assert np.isnan(got[name][1:5]).all() and np.isfinite(got[name][[0, 5]]).all()
    assert np.isnan(got["logprob"][[1, 2, 4]]).all() and got["logprob"][3] == 0
    assert np.isnan(got["top_logprob"][1:5]).all()
    assert got["top_index"][1, 0] == 7 and got["top_index"][2, 0] == cols - 1 and got["top_index"][3, 0] == 0
    np.testing.assert_array_equal(got["top_index"][4], [9, -1, -1, -1])
    ok = [0, 5]
    _, _, _, _, idx, _, _ = ref.forward(x[ok], 1.0, target[ok], 4)
    np.testing.assert_array_equal(got["top_index"][ok], idx)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_large_logits_and_small_temperatures(kind):
    """Differences count, not the size: logits around 1e4, and scales that take products out of the range."""
    rng = np.random.default_rng(6)
    x = as_held(1e4 + 64 * rng.integers(-2, 2, (3, 3000)).astype(float), kind)
    check(x, kind, 0.01, np.array([0, 1, 2]), 4)
    x = as_held(rng.standard_normal((3, 3000)), kind)
    check(x, kind, 1e4, np.array([0, 1, 2]), 4)
    got = forward(as_held(np.array([[-3e38, 1.0, 2.0, -3e38]]), kind), kind, 4.0, np.array([0]), 3)
    assert got["logprob"][0] == -np.inf and got["top_logprob"][0, 2] == -np.inf and got["top_index"][0, 2] == 0
    assert np.isfinite(got["entropy"][0])


def back(x, kind, scale, target, dlp, dh, ld=None, ldd=None, packed=None, wide=True, alias=False, both=True):
    rows, cols = x.shape
    code, tt = WIDE[kind]
    lse, _, entropy, *_ = ref.forward(x, scale, target, 1)
    lse, entropy = np.float32(lse).astype(np.float64), np.float32(entropy).astype(np.float64)
    f = lambda a: torch.from_numpy(np.float32(a)).cuda()
    tx, tt_ = up(x, tt, ld), torch.from_numpy(target).cuda()
    d = mx.LogprobDesc.make(rows, cols, scale=scale, x_type=code, ldx=ld, ldd=ldd, q_type=PACKED[packed or "e5m2"][0])
    out = {}
    if wide:
        out["dx"] = tx if alias else torch.full((rows, ldd or cols), 7.0, dtype=tt, device="cuda")[:, :cols]
    if packed:
        t = PACKED[packed][0]
        out["row"] = (mx.empty_packed(rows, cols, t), mx.empty_scales(mx.BLOCK_ROW, rows, cols))
        out["col"] = (mx.empty_packed(rows, cols, t), mx.empty_scales(mx.BLOCK_COL, rows, cols))
    given = dict(dlogprob=f(dlp)) if both else {}
    mx.logprob_bprop(d, tx, tt_, f(lse), entropy=f(entropy), dentropy=f(dh), **given, **out)
    assert mx.last_device_status() == mx.OK
    want, tol = ref.gradient(x, scale, target, lse, dlp if both else 0 * dlp, entropy, dh)
    return out, want, tol


@pytest.mark.parametrize("rows,cols,pad,padd", [(1, 1, 0, 0), (2, 5, 0, 0), (3, 128, 0, 0), (5, 131, 0, 0), (4, 1000, 8, 0), (130, 257, 0, 3),
                                                (3, 8200, 0, 0), (2, 9001, 0, 0), (140, 2049, 1, 1), (2, 30000, 0, 0)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_gradient(rows, cols, pad, padd, kind):
    rng = np.random.default_rng(rows + cols)
    x = logits(rng, rows, cols, kind)
    if rows > 2:
        x[1] = -np.inf                       # nothing left
    target = rng.integers(0, cols, rows)
    target[::4] = -1
    dlp, dh = np.float32(rng.standard_normal(rows)).astype(float), np.float32(rng.standard_normal(rows)).astype(float)
    for scale in (1.0, 0.75):
        out, want, tol = back(x, kind, scale, target, dlp, dh, cols + pad, cols + padd)
        within(down(out["dx"]), want, tol, kind)
        if rows > 2:
            assert np.all(down(out["dx"])[1] == 0)
    out2, _, _ = back(x, kind, 0.75, target, dlp, dh, cols + pad, cols + pad, alias=True)
    assert torch.equal(out2["dx"], out["dx"])
    out3, want3, tol3 = back(x, kind, 1.0, target, dlp, dh, both=False)
    within(down(out3["dx"]), want3, tol3, kind)


@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (3, 130, 0), (129, 127, 0), (128, 256, 8), (260, 1000, 3), (150, 2056, 0)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("packed", ["e4m3", "e5m2"])
def test_packed_gradient(rows, cols, pad, kind, packed):
    rng = np.random.default_rng(rows + cols)
    x = logits(rng, rows, cols, kind)
    if rows > 2:
        x[1] = -np.inf
    target = rng.integers(0, cols, rows)
    target[::4] = cols + 5
    dlp, dh = np.float32(rng.standard_normal(rows)).astype(float), np.float32(rng.standard_normal(rows)).astype(float)
    out, want, tol = back(x, kind, 1.0, target, dlp, dh, cols + pad, packed=packed)
    within(down(out["dx"]), want, tol, kind)
    near_rows(*out["row"], want, tol, packed)
    q, s = out["col"]
    near_rows(q.view(torch.uint8).t().contiguous().view(q.dtype), s, want.T, tol.T, packed)
    # the packed forms alone
    out2, _, _ = back(x, kind, 1.0, target, dlp, dh, cols + pad, packed=packed, wide=False)
    for a, b in zip((*out["row"], *out["col"]), (*out2["row"], *out2["col"])):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_gradient_of_rows_that_are_not_finite_stays_in_its_row():
    x = np.random.default_rng(0).standard_normal((3, 1000))
    x[1, 5] = np.nan
    t = torch.from_numpy(x).float().cuda()
    lse, h = torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
    d = mx.LogprobDesc.make(3, 1000, x_type=mx.DTYPE_F32)
    mx.logprob_fprop(d, t, lse=lse, entropy=h)
    dx = torch.empty_like(t)
    one = torch.ones(3, device="cuda")
    mx.logprob_bprop(d, t, torch.zeros(3, dtype=torch.int64, device="cuda"), lse, dlogprob=one, entropy=h, dentropy=one, dx=dx)
    assert bool(torch.isnan(dx[1]).all()) and bool(torch.isfinite(dx[[0, 2]]).all())
    row, col = (mx.empty_packed(3, 1000), mx.empty_scales(mx.BLOCK_ROW, 3, 1000)), (mx.empty_packed(3, 1000), mx.empty_scales(mx.BLOCK_COL, 3, 1000))
    d2 = mx.LogprobDesc.make(3, 1000, x_type=mx.DTYPE_F32, q_type=mx.DTYPE_E4M3)
    mx.logprob_bprop(d2, t, torch.zeros(3, dtype=torch.int64, device="cuda"), lse, dlogprob=one, entropy=h, dentropy=one, row=row, col=col)
    for q, _ in (row, col):
        assert np.isnan(down(q)[1]).all() and np.isfinite(down(q)[[0, 2]]).all()


@pytest.mark.parametrize("packed", [False, True])
def test_gradient_of_tokens_that_are_nearly_certain(packed):
    """dlogprob (1 - p) where p is near 1: relative to itself (ln p has one rounding, exp(ln p) - 1 a unit in its last place and the
    product one), not to p."""
    rows, cols = 16, 264
    x = torch.zeros(rows, cols, device="cuda")
    tok = torch.arange(rows, device="cuda") * 16
    x[torch.arange(rows), tok] = 4.0 + torch.arange(rows, device="cuda") * 1.5
    lse = torch.logsumexp(x.double(), 1).float()
    d = mx.LogprobDesc.make(rows, cols, x_type=mx.DTYPE_F32)
    dx, one = torch.empty_like(x), torch.ones(rows, device="cuda")
    more = dict(row=(mx.empty_packed(rows, cols, mx.DTYPE_E5M2), mx.empty_scales(mx.BLOCK_ROW, rows, cols))) if packed else {}
    mx.logprob_bprop(d, x, tok, lse, dlogprob=one, dx=dx, **more)
    got = down(dx)[np.arange(rows), tok.cpu().numpy()]
    want = -np.expm1(down(x)[np.arange(rows), tok.cpu().numpy()] - down(lse))
    assert np.all(np.abs(got - want) <= 2.0 ** -21 * np.abs(want))


def test_gradient_against_differences():
    rows, cols, step, scale = 3, 50, 1e-2, 0.8
    rng = np.random.default_rng(2)
    x = np.float32(rng.standard_normal((rows, cols)))
    target, dlp, dh = np.array([4, -1, 49]), rng.standard_normal(rows), rng.standard_normal(rows)

    def loss(x):
        got = forward(x.astype(float), "f32", scale, target)
        return float((got["logprob"] * dlp).sum() + (got["entropy"] * dh).sum())

    out, _, _ = back(x.astype(float), "f32", scale, target, np.float32(dlp).astype(float), np.float32(dh).astype(float))
    # step^2 / 6 times a third derivative of a few units, and 12 results within 1e-6 over 2 step
    tol = 10 * step * step / 6 + 12e-6 / (2 * step)
    for at in rng.choice(x.size, 20, replace=False):
        hi, lo = x.copy(), x.copy()
        hi.flat[at] += step
        lo.flat[at] -= step
        width = float(hi.flat[at]) - float(lo.flat[at])
        assert abs((loss(hi) - loss(lo)) / width - down(out["dx"]).flat[at]) <= tol


def test_rows_beyond_32_bit_offsets():
    rows, cols, ld = 3, 1001, (1 << 30) + 24
    flat = torch.zeros((rows - 1) * ld + cols, dtype=torch.bfloat16, device="cuda")
    x = flat.as_strided((rows, cols), (ld, 1))
    x.copy_(torch.randn(rows, cols, device="cuda"))
    d = mx.LogprobDesc.make(rows, cols, top=2, ldx=ld)
    lse, h, at = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, 2, dtype=torch.int32, device="cuda")
    mx.logprob_fprop(d, x, lse=lse, entropy=h, top_index=at)
    near = torch.logsumexp(x.double(), 1)
    assert float((lse.double() - near).abs().max()) <= 1e-4
    assert torch.equal(at[:, 0].long(), x.float().argmax(1))
    dx, want = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda"), None
    one, tok = torch.ones(rows, device="cuda"), torch.zeros(rows, dtype=torch.int64, device="cuda")
    mx.logprob_bprop(d, x, tok, lse, dlogprob=one, dx=dx)
    want = -torch.softmax(x.double(), 1)
    want[:, 0] += 1
    assert float((dx.double() - want).abs().max()) <= 2.0 ** -8
