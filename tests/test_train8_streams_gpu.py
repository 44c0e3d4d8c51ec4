"""Products on several streams at once: clusters of several CTAs and pairs of SMs that allocate tensor memory, next
to the convolution kernels that do."""
import pytest
import torch

import paper_1501_06633_b200 as mx

pytestmark = pytest.mark.gpu


class Product:
    def __init__(self, M, N, K, cols, pair, split, seed, c_type=mx.DTYPE_F32, f32_scales=False):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.options = (("GEMM8_COLS", cols), ("GEMM8_PAIR", pair), ("GEMM8_SPLIT", split), ("GEMM8_SWAP", 0))
        sides = []
        for n in (M, N):
            q, s = mx.empty_packed(n, K), mx.empty_scales(mx.BLOCK_ROW, n, K)
            mx.quant8(mx.Quant8Desc.make(n, K, x_type=mx.DTYPE_F32), torch.randn(n, K, device="cuda", generator=gen), row=(q, s))
            sides += [q, s.to(torch.float32) if f32_scales else s]
        kind = mx.DTYPE_F32 if f32_scales else mx.DTYPE_E8M0
        self.desc = mx.Gemm8Desc.make(M, N, K, c_type=c_type, b_block=mx.BLOCK_ROW, a_scale_type=kind, b_scale_type=kind)
        self.sides, self.c = sides, torch.zeros(M, N, device="cuda")

    def run(self, stream=None):
        for name, v in self.options:
            mx.set_option(name, v)
        mx.gemm8(self.desc, *self.sides, self.c, stream=stream)


def test_clusters_on_several_streams():
    works = [Product(700, 900, 256, 128, -1, 2, 1), Product(700, 900, 384, 64, -1, 2, 2), Product(600, 800, 1024, 16, -1, 8, 3),
             Product(2500, 2500, 128, 128, 1, 1, 4), Product(2500, 2500, 256, 256, 1, 1, 5),
             Product(700, 900, 256, 256, 0, 2, 6, f32_scales=True)]
    works[5].options = (("GEMM8_COLS", 256), ("GEMM8_SPLIT", 2), ("GEMM8_SWAP", 0), ("GEMM8_PAIR", -1))
    d = mx.ConvDesc.make(64, 9, 9, 8, 256, 3, 1, 1, 1.0)
    gen = torch.Generator(device="cuda").manual_seed(7)
    maps = torch.randn(mx.conv_in_elems(d), device="cuda", generator=gen)
    filt = torch.randn(mx.conv_filt_elems(d), device="cuda", generator=gen)
    out = torch.empty(mx.conv_out_elems(d), device="cuda")
    mx.conv_fprop_tf32(d, maps, filt, out)
    want = [out.clone()]
    for w in works:
        w.run()
        torch.cuda.synchronize()
        want.append(w.c.clone())
        w.c.zero_()
    out.zero_()
    assert mx.last_device_status() == mx.OK
    streams = [torch.cuda.Stream() for _ in range(len(works) + 1)]
    torch.cuda.synchronize()
    for _ in range(40):
        mx.conv_fprop_tf32(d, maps, filt, out, stream=streams[0])
        for w, s in zip(works, streams[1:]):
            w.run(s)
    torch.cuda.synchronize()
    assert mx.last_device_status() == mx.OK
    for got, w in zip([out] + [w.c for w in works], want):
        assert torch.equal(got, w)
