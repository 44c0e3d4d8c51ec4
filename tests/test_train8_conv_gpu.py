"""A 1x1 convolution as a product of 8-bit matrices: maps [channels][positions x images] and filters
[channels][filters] are read as the convolution kernels store them, in blocks along the channels."""
import pytest
import torch

import paper_1501_06633_b200 as mx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("images,side,channels,filters", [(16, 5, 48, 64), (64, 7, 200, 132), (32, 9, 256, 96)])
def test_one_by_one_convolution(images, side, channels, filters):
    gen = torch.Generator(device="cuda").manual_seed(channels)
    d = mx.ConvDesc.make(images, side, side, channels, filters, 1, 1, 0, 1.0)
    positions = side * side * images
    maps = torch.randn(channels, positions, device="cuda", generator=gen)
    filt = torch.randn(channels, filters, device="cuda", generator=gen) / channels ** 0.5
    packed = []
    for x in (filt, maps):
        rows, cols = x.shape
        q, s = mx.empty_packed(rows, cols), mx.empty_scales(mx.BLOCK_COL, rows, cols)
        desc = mx.Quant8Desc.make(rows, cols, x_type=mx.DTYPE_F32)
        mx.quant8(desc, x, col=(q, s))
        back = torch.empty_like(x)
        mx.dequant8(desc, q, s, back, mx.BLOCK_COL)
        packed.append((q, s, back))
    (qf, sf, f), (qm, sm, m) = packed
    out = torch.empty(filters, positions, device="cuda")
    mx.gemm8(mx.Gemm8Desc.make(filters, positions, channels, c_type=mx.DTYPE_F32, a_major=mx.MAJOR_MN, b_major=mx.MAJOR_MN,
                               b_block=mx.BLOCK_COL), qf, sf, qm, sm, out)
    want = torch.empty(mx.conv_out_elems(d), device="cuda")
    mx.conv_fprop(d, m, f, want)                  # the fp32 convolution of what the packed operands stand for
    assert mx.last_device_status() == mx.OK
    # two fp32 sums of the same products: one rounding a term there, 2^-23 of the running sum a block and MMA here
    tol = (channels * 2.0 ** -24 + (128 + 2) * 2.0 ** -23) * (f.abs().t() @ m.abs())
    assert bool(((out - want.view_as(out)).abs() <= tol).all())
