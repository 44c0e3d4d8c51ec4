"""A feed-forward block of a language model, trained and served with the 8-bit operators.

    y = layer_norm(x);  h = y W1^T;  a = silu(h_gate) h_up;  out = x + a W2^T

What is kept between the forward and the backward pass is in 8 bits: the packed input of the layer
norm, the packed operands of both products and the packed inputs of the activation (about 1 byte
per value instead of 2).  Weights are packed once per update, in 128 x 128 blocks, and serve the
forward pass and the input gradient as they lie; the weight gradients read the tokens' operands
packed again along the tokens.

    python examples/feed_forward8.py             trains on a synthetic task, then times one token

`conv_filter_gradient` does the same for this library's convolution: maps kept in 8 bits, unpacked
for the BF16 filter gradient.
"""
import os
import sys
import time

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_1501_06633_b200 as mx  # noqa: E402


def scales(block, rows, cols):
    return mx.empty_scales(block, rows, cols)


class Linear8:
    """A weight [outer][inner] with its packed form, and the three products of a linear layer."""

    def __init__(self, outer, inner, gen):
        self.outer, self.inner = outer, inner
        self.master = torch.randn(outer, inner, device="cuda", generator=gen) / inner ** 0.5
        self.q = mx.empty_packed(outer, inner)
        self.s = scales(mx.BLOCK_TILE, outer, inner)
        self.pack()

    def pack(self):
        mx.quant8(mx.Quant8Desc.make(self.outer, self.inner, x_type=mx.DTYPE_F32), self.master, tile=(self.q, self.s))

    def forward(self, q, s, out):
        """out [tokens][outer] = x W^T from packed rows of x."""
        d = mx.Gemm8Desc.make(q.shape[0], self.outer, self.inner, lda=q.stride(0), ldb=self.q.stride(0))
        mx.gemm8(d, q, s, self.q, self.s, out)

    def input_gradient(self, q, s, out):
        """out [tokens][inner] = dy W from packed rows of dy, with the weights as they are stored."""
        d = mx.Gemm8Desc.make(q.shape[0], self.inner, self.outer, a_type=mx.DTYPE_E5M2, b_major=mx.MAJOR_MN,
                              lda=q.stride(0), ldb=self.q.stride(0))
        mx.gemm8(d, q, s, self.q, self.s, out)

    def weight_gradient(self, qd, sd, qx, sx):
        """dW [outer][inner] = dy^T x from columns of both."""
        out = torch.empty(self.outer, self.inner, device="cuda")
        d = mx.Gemm8Desc.make(self.outer, self.inner, qd.shape[0], a_type=mx.DTYPE_E5M2, c_type=mx.DTYPE_F32,
                              a_major=mx.MAJOR_MN, b_major=mx.MAJOR_MN, b_block=mx.BLOCK_COL, lda=qd.stride(0), ldb=qx.stride(0))
        mx.gemm8(d, qd, sd, qx, sx, out)
        return out


def pack_gradient(g):
    """Rows (for the input gradient) and columns (for the weight gradient) of a gradient, in one reading."""
    r, c = g.shape
    row = mx.empty_packed(r, c, mx.DTYPE_E5M2), scales(mx.BLOCK_ROW, r, c)
    col = mx.empty_packed(r, c, mx.DTYPE_E5M2), scales(mx.BLOCK_COL, r, c)
    mx.quant8(mx.Quant8Desc.make(r, c, q_type=mx.DTYPE_E5M2), g, row=row, col=col)
    return row, col


def columns_of(q, s):
    """A matrix packed in rows, packed again in columns."""
    r, c = q.shape
    col = mx.empty_packed(r, c), scales(mx.BLOCK_COL, r, c)
    mx.quant8(mx.Quant8Desc.make(r, c, x_type=mx.DTYPE_E4M3, ldx=q.stride(0) if r > 1 else None), q, col=col, x_scale=s)
    return col


class FeedForward8:
    def __init__(self, width, inner, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.width, self.inner = width, inner
        self.gamma, self.beta = torch.ones(width, device="cuda"), torch.zeros(width, device="cuda")
        self.up, self.down = Linear8(2 * inner, width, gen), Linear8(width, inner, gen)
        self.kept = None

    def forward(self, x, train=True):
        t, w, f = x.shape[0], self.width, self.inner
        ln = mx.LayerNormDesc.make(t, w)
        y = mx.empty_packed(t, w), scales(mx.BLOCK_ROW, t, w)
        stats = torch.empty(2, t, device="cuda")
        cx = (mx.empty_packed(t, w), scales(mx.BLOCK_ROW, t, w)) if train else None
        mx.layer_norm_fprop(ln, x, self.gamma, self.beta, mean=stats[0], rstd=stats[1], packed=y, checkpoint=cx)
        h = torch.empty(t, 2 * f, dtype=torch.bfloat16, device="cuda")
        self.up.forward(*y, h)
        a = mx.empty_packed(t, f), scales(mx.BLOCK_ROW, t, f)
        blocks = -(-f // 128)
        ch = (mx.empty_packed(t, 2 * f), torch.empty(2 * blocks, t, dtype=torch.uint8, device="cuda")) if train else None
        mx.act8_fprop(mx.Act8Desc.make(t, f, ldc=ch[0].stride(0) if train else None), h, packed=a, checkpoint=ch)
        out = torch.empty_like(x)
        self.down.forward(*a, out)
        self.kept = (y, stats, cx, a, ch) if train else None
        return x + out

    def backward(self, dout):
        """Gradients by name, from what forward kept."""
        (y, stats, (cx, scx), a, (ch, sch)), (t, w), f = self.kept, dout.shape, self.inner
        row, col = pack_gradient(dout)
        grads = {"down": self.down.weight_gradient(*col, *columns_of(*a))}
        da = torch.empty(t, f, dtype=torch.bfloat16, device="cuda")
        self.down.input_gradient(*row, da)
        dh = torch.empty(t, 2 * f, dtype=torch.bfloat16, device="cuda")
        mx.act8_bprop(mx.Act8Desc.make(t, f, h_type=mx.DTYPE_E4M3, ldc=ch.stride(0)), da, ch, dh, h_scale=sch)
        row, col = pack_gradient(dh)
        grads["up"] = self.up.weight_gradient(*col, *columns_of(*y))
        dy = torch.empty(t, w, dtype=torch.bfloat16, device="cuda")
        self.up.input_gradient(*row, dy)
        d = mx.LayerNormDesc.make(t, w, x_type=mx.DTYPE_E4M3, y_type=mx.DTYPE_BF16, ldx=cx.stride(0))
        ws = torch.empty(max(16, mx.layer_norm_bprop_workspace(d)), dtype=torch.uint8, device="cuda")
        dx = torch.empty_like(dy)
        grads["gamma"], grads["beta"] = torch.empty(w, device="cuda"), torch.empty(w, device="cuda")
        mx.layer_norm_bprop(d, dy, cx, self.gamma, stats[0], stats[1], dx, grads["gamma"], grads["beta"], ws, x_scale=scx)
        grads["x"] = dx + dout
        return grads

    def update(self, grads, rate):
        self.gamma -= rate * grads["gamma"]
        self.beta -= rate * grads["beta"]
        for layer, name in ((self.up, "up"), (self.down, "down")):
            layer.master -= rate * grads[name]
            layer.pack()


def conv_filter_gradient(desc, maps, dout):
    """The filter gradient of a convolution whose maps were kept in 8 bits: rows of the packed matrix
    are the map positions, columns the images."""
    rows, images = desc.Nc * desc.Hi * desc.Wi, desc.Nb
    q, s = mx.empty_packed(rows, images), scales(mx.BLOCK_ROW, rows, images)
    mx.quant8(mx.Quant8Desc.make(rows, images), maps.view(rows, images), row=(q, s))           # forward pass: kept
    back = torch.empty(rows, images, dtype=torch.bfloat16, device="cuda")
    mx.dequant8(mx.Quant8Desc.make(rows, images, ldq=q.stride(0)), q, s, back, mx.BLOCK_ROW)   # backward pass: unpacked
    dfilt = torch.empty(mx.conv_filt_elems(desc), device="cuda")
    ws = torch.empty(max(16, mx.conv_bprop_filter_workspace(desc, mx.KERNEL_BF16)), dtype=torch.uint8, device="cuda")
    mx.conv_bprop_filter(desc, back, dout, dfilt, ws, mx.KERNEL_BF16)
    return dfilt


def main():
    torch.manual_seed(0)
    tokens, width, inner = 4096, 1024, 2048
    block, teacher = FeedForward8(width, inner, seed=1), FeedForward8(width, inner, seed=2)
    x = torch.randn(tokens, width, device="cuda").to(torch.bfloat16)
    goal = teacher.forward(x, train=False).float()
    for step in range(31):
        out = block.forward(x).float()
        diff = out - goal
        loss = float((diff * diff).mean())
        block.update(block.backward((2 * diff / width).to(torch.bfloat16)), rate=2e-2 / tokens * width)
        if step % 5 == 0:
            print("step %2d  loss %.4f" % (step, loss))
    one = x[:1].contiguous()
    for _ in range(3):
        block.forward(one, train=False)
    torch.cuda.synchronize()
    t = time.perf_counter()
    for _ in range(100):
        block.forward(one, train=False)
    torch.cuda.synchronize()
    print("one token: %.1f us" % ((time.perf_counter() - t) * 1e4))
    assert mx.last_device_status() == mx.OK


if __name__ == "__main__":
    main()
