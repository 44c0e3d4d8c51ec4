"""Calls in a row without synchronising between them.  Kernels may be resident before the ones in front of them
have finished, and buffers are written and read again within a chain, so a value kept from before a
buffer was rewritten would show in the chain's results."""
import pytest
import torch

import paper_1501_06633_b200 as mx

pytestmark = pytest.mark.gpu


class Chain:
    """A chain over two buffers [rows][width] that are read and rewritten in turn: layer norm, activation,
    packing, product, unpacking, and both backward passes."""

    def __init__(self, rows, width, seed):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.rows, self.width = rows, width
        new = lambda *s: torch.randn(*s, device="cuda", generator=gen)
        self.buf = [torch.zeros(rows, width, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        self.dx = torch.zeros_like(self.buf[0])
        self.start = [new(rows, width).to(torch.bfloat16) for _ in range(4)]
        self.gamma, self.beta = 1 + 0.2 * new(width), 0.3 * new(width)
        self.q, self.s = mx.empty_packed(rows, width), mx.empty_scales(mx.BLOCK_ROW, rows, width)
        self.w, self.ws = mx.empty_packed(width, width), mx.empty_scales(mx.BLOCK_TILE, width, width)
        mx.quant8(mx.Quant8Desc.make(width, width, x_type=mx.DTYPE_F32), new(width, width) / width ** 0.5, tile=(self.w, self.ws))
        self.mean, self.rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        self.dgamma, self.dbeta = torch.empty(width, device="cuda"), torch.empty(width, device="cuda")
        self.ln, self.act = mx.LayerNormDesc.make(rows, width), mx.Act8Desc.make(rows, width, gated=False)
        self.pack, self.product = mx.Quant8Desc.make(rows, width), mx.Gemm8Desc.make(rows, width, width)
        self.scratch = torch.empty(mx.layer_norm_bprop_workspace(self.ln), dtype=torch.uint8, device="cuda")

    def run(self, turns, after):
        a, b = self.buf
        steps = (
            lambda: mx.layer_norm_fprop(self.ln, a, self.gamma, self.beta, y=b, mean=self.mean, rstd=self.rstd),
            lambda: mx.quant8(self.pack, b, row=(self.q, self.s)),
            lambda: mx.gemm8(self.product, self.q, self.s, self.w, self.ws, a),
            lambda: mx.act8_fprop(self.act, a, a=b, packed=(self.q, self.s)),
            lambda: mx.dequant8(self.pack, self.q, self.s, a, mx.BLOCK_ROW),
            lambda: mx.layer_norm_fprop(self.ln, a, mean=self.mean, rstd=self.rstd, packed=(self.q, self.s)),
            lambda: mx.layer_norm_bprop(self.ln, b, a, self.gamma, self.mean, self.rstd, self.dx, self.dgamma, self.dbeta, self.scratch),
            lambda: mx.act8_bprop(self.act, self.dx, b, a),
            lambda: mx.layer_norm_fprop(self.ln, a, self.dgamma, self.dbeta, y=b),
            lambda: mx.act8_fprop(self.act, b, a=a),
        )
        for _ in range(turns):
            for step in steps:
                step()
                after()

    def results(self):
        return [t.clone() for t in (*self.buf, self.q.view(torch.uint8), self.s.view(torch.uint8), self.mean, self.rstd, self.dgamma,
                                    self.dbeta, self.dx)]


@pytest.mark.parametrize("rows,width", [(16, 128), (64, 512), (200, 1040), (700, 2048)])
def test_chains_give_what_synchronised_calls_give(rows, width):
    turns = 4
    chain = Chain(rows, width, seed=rows)
    want = []
    for start in chain.start:
        chain.buf[0].copy_(start)
        torch.cuda.synchronize()
        chain.run(turns, torch.cuda.synchronize)
        want.append(chain.results())
    assert not torch.equal(want[0][0], want[1][0])
    assert all(bool(torch.isfinite(t.float()).all()) for t in (want[0][0], want[0][6]))
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        chain.run(turns, lambda: None)
    for again in range(24):
        k = again % len(want)
        chain.buf[0].copy_(chain.start[k])
        if again % 2:
            graph.replay()
        else:
            chain.run(turns, lambda: None)
        torch.cuda.synchronize()
        for got, w in zip(chain.results(), want[k]):
            assert torch.equal(got, w), (again, k)
    assert mx.last_device_status() == mx.OK
