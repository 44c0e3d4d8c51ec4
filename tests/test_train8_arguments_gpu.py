"""What the Python calls of the 8-bit operators answer to arguments that their descriptors do not cover."""
import pytest
import torch

import paper_1501_06633_b200 as mx

pytestmark = pytest.mark.gpu


def e8(*s):
    return torch.zeros(*s, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("code", [6, 9, 100, -1])
def test_types_that_do_not_exist(code):
    """As for every other descriptor field: an error of type or value, not of an index."""
    x, v = torch.zeros(4, 128, device="cuda"), torch.zeros(128, device="cuda")
    r = torch.zeros(4, device="cuda")
    f = mx.DTYPE_F32
    refused = pytest.raises((TypeError, ValueError, mx.MaxdnnError))
    with refused:
        mx.layer_norm_fprop(mx.LayerNormDesc.make(4, 128, x_type=f, w_type=code), x, v, v, y=x)
    with refused:
        mx.layer_norm_bprop(mx.LayerNormDesc.make(4, 128, x_type=f, w_type=code), x, x, v, r, r, torch.empty_like(x))
    with refused:
        mx.gemm8(mx.Gemm8Desc.make(4, 4, 128, c_type=f, b_block=mx.BLOCK_ROW, a_scale_type=code), e8(4, 128), e8(1, 4), e8(4, 128),
                 e8(1, 4), torch.zeros(4, 4, device="cuda"))
    with refused:
        mx.quant8(mx.Quant8Desc.make(4, 128, x_type=f, q_type=code), x, row=(e8(4, 128), e8(1, 4)))
    with refused:
        mx.dequant8(mx.Quant8Desc.make(4, 128, x_type=code), e8(4, 128), e8(1, 4), x)
    with refused:
        mx.act8_fprop(mx.Act8Desc.make(4, 64, x_type=code), x, a=torch.zeros(4, 64, device="cuda"))
    with refused:
        mx.act8_bprop(mx.Act8Desc.make(4, 64, x_type=f, h_type=code), torch.zeros(4, 64, device="cuda"), x, torch.empty_like(x))
    assert mx.last_device_status() == mx.OK


@pytest.mark.parametrize("block", [3, 7, -1])
def test_blocks_that_do_not_exist(block):
    refused = pytest.raises((TypeError, ValueError, mx.MaxdnnError))
    with refused:
        mx.dequant8(mx.Quant8Desc.make(4, 128, x_type=mx.DTYPE_F32), e8(4, 128), e8(1, 4), torch.zeros(4, 128, device="cuda"), block)
    with refused:
        mx.gemm8(mx.Gemm8Desc.make(4, 4, 128, c_type=mx.DTYPE_F32, a_block=block, b_block=mx.BLOCK_ROW), e8(4, 128), e8(1, 4), e8(4, 128),
                 e8(1, 4), torch.zeros(4, 4, device="cuda"))


def test_tensors_that_do_not_fit():
    """Sizes, types and strides other than the descriptor's, values without scales, a tensor of the host."""
    x = torch.zeros(4, 128, device="cuda")
    q, s = e8(4, 128), e8(1, 4)
    d = mx.Quant8Desc.make(4, 128, x_type=mx.DTYPE_F32)
    for bad in (dict(x=x[:, :100]), dict(x=x.half()), dict(x=x.cpu()), dict(x=x.t().contiguous().t()), dict(row=(q, e8(1, 5))),
                dict(row=(q, None)), dict(row=(e8(4, 64), s)), dict(row=(q, s.float()))):
        with pytest.raises((TypeError, ValueError, mx.MaxdnnError)):
            mx.quant8(d, **{**dict(x=x, row=(q, s)), **bad})
    with pytest.raises(mx.MaxdnnError):
        mx.quant8(d, x)                                        # nothing asked for
    mx.quant8(d, x.view(-1), row=(q.view(-1), s.view(-1)))     # the same elements in another shape
    assert mx.last_device_status() == mx.OK
