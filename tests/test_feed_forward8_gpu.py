"""The example block that runs the 8-bit operators together: its gradients against the same block in
64 bits, and its training.  An E4M3 value carries a relative rounding error of up to 2^-4 (uniform: 2^-4 / sqrt(12)
of a step, about 2 % rms), an E5M2 value twice that; a gradient passes at most four packed operands and
two 16-bit roundings: 12 % rms if all add up in quadrature with the gradient packings' 4 %."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import paper_1501_06633_b200 as mx

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
spec = importlib.util.spec_from_file_location("feed_forward8", os.path.join(ROOT, "examples", "feed_forward8.py"))
ff = importlib.util.module_from_spec(spec)
spec.loader.exec_module(ff)


def exact_grads(block, x, dout):
    x = x.double().requires_grad_()
    gamma, beta = block.gamma.double().requires_grad_(), block.beta.double().requires_grad_()
    w1, w2 = block.up.master.double().requires_grad_(), block.down.master.double().requires_grad_()
    mean = x.mean(1, keepdim=True)
    y = (x - mean) / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + 1e-5) * gamma + beta
    h = y @ w1.t()
    g, u = h.split(block.inner, 1)
    out = x + (g * torch.sigmoid(g) * u) @ w2.t()
    out.backward(dout.double())
    return out.detach(), {"x": x.grad, "gamma": gamma.grad, "beta": beta.grad, "up": w1.grad, "down": w2.grad}


@pytest.mark.parametrize("tokens,width,inner", [(256, 256, 384), (300, 200, 150), (1, 128, 256)])
def test_block_against_64_bits(tokens, width, inner):
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    block = ff.FeedForward8(width, inner, seed=3)
    block.gamma += 0.2 * torch.randn(width, device="cuda", generator=gen)
    x = torch.randn(tokens, width, device="cuda", generator=gen).to(torch.bfloat16)
    dout = torch.randn(tokens, width, device="cuda", generator=gen).to(torch.bfloat16)
    out = block.forward(x)
    grads = block.backward(dout)
    assert mx.last_device_status() == mx.OK
    want, exact = exact_grads(block, x, dout)
    rel = lambda a, b: float((a.double() - b).norm() / b.norm())
    assert rel(out, want) <= 0.06
    for name, g in exact.items():
        assert rel(grads[name], g) <= 0.12, name
    assert torch.equal(block.forward(x, train=False), out)


def test_block_learns():
    block, teacher = ff.FeedForward8(256, 512, seed=1), ff.FeedForward8(256, 512, seed=2)
    x = torch.randn(1024, 256, device="cuda", generator=torch.Generator(device="cuda").manual_seed(0)).to(torch.bfloat16)
    goal = teacher.forward(x, train=False).float()
    losses = []
    for _ in range(15):
        diff = block.forward(x).float() - goal
        losses.append(float((diff * diff).mean()))
        block.update(block.backward((2 * diff / 256).to(torch.bfloat16)), rate=2e-2 / 1024 * 256)
    assert losses[-1] < 0.8 * losses[0]


def test_convolution_from_packed_maps():
    """Maps kept in 8 bits for the filter gradient: the maps' rounding (2 % rms) is what it may differ by."""
    d = mx.ConvDesc.make(128, 9, 9, 32, 64, 3, 1, 1, 1.0)
    gen = torch.Generator(device="cuda").manual_seed(1)
    maps = torch.randn(mx.conv_in_elems(d), device="cuda", generator=gen).to(torch.bfloat16)
    dout = torch.randn(mx.conv_out_elems(d), device="cuda", generator=gen).to(torch.bfloat16)
    got = ff.conv_filter_gradient(d, maps, dout)
    want = torch.empty_like(got)
    ws = torch.empty(max(16, mx.conv_bprop_filter_workspace(d, mx.KERNEL_BF16)), dtype=torch.uint8, device="cuda")
    mx.conv_bprop_filter(d, maps, dout, want, ws, mx.KERNEL_BF16)
    assert mx.last_device_status() == mx.OK
    assert float((got - want).norm() / want.norm()) <= 0.04
    assert not np.isnan(float(got.sum()))
