"""The kernel instances that training batches run: layer norm by warps and groups of warps, backward with
more rows a CTA than its statistics are fetched at once, products of several accumulator chunks on two-SM
tiles, results stored by bulk copies.  Tolerances as in test_train8_gpu.py and test_train8_norm_gpu.py."""
import numpy as np
import pytest
import torch

import paper_1501_06633_b200 as mx
import train8_ref as ref
from test_train8_gpu import PACKED, SUM_TOL, WAYS, WIDE, as_held, bytes_of, data, down, near_packed, run_gemm, same, up, within

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ layer norm
@pytest.mark.parametrize("cols", [200, 300, 512, 600, 1024, 1500, 2048, 3000, 4096, 5000])
@pytest.mark.parametrize("kind,qt,weights", [("f32", "e4m3", "f32"), ("bf16", "e4m3", "f32"), ("bf16", "e5m2", "bf16"), ("f16", "e4m3", "f16")])
def test_forward_of_many_rows(cols, kind, qt, weights):
    """More rows than four per SM, and more than the CTAs of a device hold at once: y, statistics and both
    packings in one call."""
    rows = 700 if cols <= 2048 else 1300
    rng = np.random.default_rng(cols)
    x = as_held(3.0 * data(rng, rows, cols, False) + 2.0, kind)
    gamma, beta = as_held(rng.uniform(-2, 2, cols), weights), as_held(rng.standard_normal(cols), weights)
    want, mean, rstd = ref.layer_norm(x, gamma, beta, 1e-5)
    code, tt = WIDE[kind]
    d = mx.LayerNormDesc.make(rows, cols, x_type=code, w_type=WIDE[weights][0], q_type=PACKED[qt][0])
    y = torch.empty(rows, cols, dtype=tt, device="cuda")
    m, r = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    q, c = (mx.empty_packed(rows, cols, PACKED[qt][0]) for _ in range(2))
    s, sc = (mx.empty_scales(mx.BLOCK_ROW, rows, cols) for _ in range(2))
    mx.layer_norm_fprop(d, up(x, tt), up(gamma, WIDE[weights][1]), up(beta, WIDE[weights][1]), y=y, mean=m, rstd=r, packed=(q, s),
                        checkpoint=(c, sc))
    size = np.abs(x).mean(1)
    assert np.all(np.abs(down(m) - mean) <= SUM_TOL * size)
    rel = 2 * SUM_TOL + 4 * SUM_TOL * size * rstd
    assert np.all(np.abs(down(r) - rstd) <= rel * rstd)
    tol = (rel[:, None] + 2.0 ** -22) * (np.abs((want - beta)) + np.abs(gamma)) + 2.0 ** -22 * np.abs(want)
    within(down(y), want, tol, kind)
    some = np.r_[0:40, rows // 2:rows // 2 + 40, rows - 40:rows]      # (the plain packing goes block by block)
    wq, ws = ref.pack(x[some], "row", qt)
    same(down(c)[some], wq)
    np.testing.assert_array_equal(bytes_of(sc)[:, some], ws)
    at = torch.from_numpy(some).cuda()
    near_packed(q.view(torch.uint8)[at].view(q.dtype), s.view(torch.uint8)[:, at].contiguous().view(s.dtype), want[some], tol[some], qt)
    # the packings alone give the same bytes, and so does every repetition
    for _ in range(3):
        again = [torch.zeros_like(t.view(torch.uint8)) for t in (q, s, c, sc)]
        mx.layer_norm_fprop(d, up(x, tt), up(gamma, WIDE[weights][1]), up(beta, WIDE[weights][1]),
                            packed=(mx.empty_packed(rows, cols, PACKED[qt][0]), again[1]))
        two = mx.empty_packed(rows, cols, PACKED[qt][0]), mx.empty_packed(rows, cols, PACKED[qt][0])
        mx.layer_norm_fprop(d, up(x, tt), up(gamma, WIDE[weights][1]), up(beta, WIDE[weights][1]), packed=(two[0], again[1]),
                            checkpoint=(two[1], again[3]))
        for a, b in ((two[0], q), (two[1], c)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        assert torch.equal(again[1], s.view(torch.uint8)) and torch.equal(again[3], sc.view(torch.uint8))


def values_of(q, s):
    """A packed matrix in 64 bits on the GPU, rows of 128."""
    scale = torch.pow(2.0, s.view(torch.uint8).double() - 127).t().repeat_interleave(128, 1)[:, :q.shape[1]]
    return q.to(torch.float32).double() * scale


# rows a CTA: 592 CTAs of 128 threads, 296 of 256, 148 of 512, each with at least 33 of the rows
@pytest.mark.parametrize("rows,cols", [(700, 4096), (20000, 1032), (10000, 2056), (10000, 4096), (5000, 4104), (5200, 8192)])
@pytest.mark.parametrize("kind,packed", [("bf16", "e4m3"), ("f32", None), ("f16", "e5m2")])
def test_backward_of_many_rows(rows, cols, kind, packed):
    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    new = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    code, tt = WIDE[kind]
    x, dy = (2 * new(rows, cols) + 1).to(tt), new(rows, cols).to(tt)
    gamma = torch.rand(cols, device="cuda", generator=gen) + 0.5
    mean, rstd = x.double().mean(1).float(), (x.double().var(1, unbiased=False) + 1e-5).rsqrt().float()
    sx = None
    if packed:
        q, sx = mx.empty_packed(rows, cols, PACKED[packed][0]), mx.empty_scales(mx.BLOCK_ROW, rows, cols)
        mx.quant8(mx.Quant8Desc.make(rows, cols, x_type=code, q_type=PACKED[packed][0]), x, row=(q, sx))
        d = mx.LayerNormDesc.make(rows, cols, x_type=PACKED[packed][0], y_type=code, ldx=q.stride(0))
        v, x = values_of(q, sx), q
    else:
        d, v = mx.LayerNormDesc.make(rows, cols, x_type=code), x.double()
    dx, dg, db = torch.empty(rows, cols, dtype=tt, device="cuda"), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(mx.layer_norm_bprop_workspace(d), dtype=torch.uint8, device="cuda")
    mx.layer_norm_bprop(d, dy, x, gamma, mean, rstd, dx, dg, db, ws, x_scale=sx)
    xh, r = (v - mean.double()[:, None]) * rstd.double()[:, None], rstd.double()[:, None]
    del v
    e = dy.double() * gamma.double()
    want = r * (e - e.mean(1, keepdim=True) - xh * (e * xh).mean(1, keepdim=True))
    tol = r * SUM_TOL * (e.abs() + e.abs().mean(1, keepdim=True) + xh.abs() * (e * xh).abs().mean(1, keepdim=True))
    assert bool((dx >= (want - tol).to(tt)).all()) and bool((dx <= (want + tol).to(tt)).all())
    row_tol = (rows + 32) * 2.0 ** -24
    dyd = dy.double()
    assert bool(((dg - (dyd * xh).sum(0)).abs() <= (row_tol + 2.0 ** -23) * (dyd * xh).abs().sum(0)).all())
    assert bool(((db - dyd.sum(0)).abs() <= row_tol * dyd.abs().sum(0)).all())
    again = [torch.empty_like(t) for t in (dx, dg, db)]
    mx.layer_norm_bprop(d, dy, x, gamma, mean, rstd, *again, ws, x_scale=sx)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dg, db)))


# ------------------------------------------------------------------ products
@pytest.mark.parametrize("pair,cols", [(-1, 32), (-1, 64), (-1, 128), (1, 128), (1, 192), (1, 224), (1, 256)])
@pytest.mark.parametrize("way", ["fprop", "dgrad", "wgrad"])
@pytest.mark.parametrize("ct", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("ldc", [328, 344])
def test_results_stored_by_bulk_copies(pair, cols, way, ct, ldc):
    """Rows of C that start and end at multiples of 16 bytes, with and without a gap between them."""
    mx.set_option("GEMM8_PAIR", pair)
    mx.set_option("GEMM8_COLS", cols)
    mx.set_option("GEMM8_SPLIT", 1)
    mx.set_option("GEMM8_SWAP", 0)
    run_gemm(150, 328, 300, *WAYS[way], ct=ct, ldc=ldc, seed=cols)


def random_operand(rows, cols, scales_shape, gen):
    """E4M3 numbers of any size and sign, scales of 2^-6 to 2^6."""
    q = torch.randint(0, 256, (rows, cols), dtype=torch.uint8, device="cuda", generator=gen)
    q = torch.where((q & 0x7F) == 0x7F, 0x30, q)
    return q.view(torch.float8_e4m3fn), torch.randint(127 - 6, 127 + 7, scales_shape, dtype=torch.uint8, device="cuda", generator=gen)


def along(q, s, by_column):
    """Values in 64 bits; scales in row blocks, or in column blocks."""
    p = torch.pow(2.0, s.double() - 127)
    p = p.repeat_interleave(128, 0)[:q.shape[0]] if by_column else p.t().repeat_interleave(128, 1)[:, :q.shape[1]]
    return q.to(torch.float32).double() * p


@pytest.mark.parametrize("pair,cols", [(-1, 16), (-1, 64), (-1, 128), (1, 128), (1, 192), (1, 224), (1, 256)])
@pytest.mark.parametrize("way", ["fprop", "wgrad"])
@pytest.mark.parametrize("ct", ["f32", "bf16"])
def test_many_tiles_of_several_chunks(pair, cols, way, ct):
    """More tiles than SMs or pairs of them; five accumulators for each tile of an fp32 result, the last of them
    short (K = 8500: 67 blocks)."""
    M, N, K = (2300, 2632, 8500) if cols > 16 else (600, 1320, 8500)
    gen = torch.Generator(device="cuda").manual_seed(cols)
    mx.set_option("GEMM8_PAIR", pair)
    mx.set_option("GEMM8_COLS", cols)
    mx.set_option("GEMM8_SPLIT", 1)
    by_column = way == "wgrad"
    blocks = -(-K // 128)
    side = []
    for n in (M, N):
        shape = (K, -(-n // 16) * 16) if by_column else (n, -(-K // 16) * 16)
        q, s = random_operand(*shape, (blocks, n), gen)
        q = q[:, :n] if by_column else q[:, :K]
        v = along(q, s, by_column)
        side.append((q, s, v.t() if by_column else v))
    (a, sa, va), (b, sb, vb) = side
    major = mx.MAJOR_MN if by_column else mx.MAJOR_K
    block = mx.BLOCK_COL if by_column else mx.BLOCK_ROW
    c = torch.empty(M, N, dtype=WIDE[ct][1], device="cuda")
    d = mx.Gemm8Desc.make(M, N, K, c_type=WIDE[ct][0], a_major=major, b_major=major, a_block=block, b_block=block, lda=a.stride(0),
                          ldb=b.stride(0))
    mx.gemm8(d, a, sa, b, sb, c)
    assert mx.last_device_status() == mx.OK
    want, tol = va @ vb.t(), (4 * (16 if ct == "f32" else blocks) + 64 + blocks) * 2.0 ** -23 * (va.abs() @ vb.abs().t())
    assert bool((c >= (want - tol).to(c.dtype)).all()) and bool((c <= (want + tol).to(c.dtype)).all())
