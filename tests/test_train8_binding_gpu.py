"""The marshalling module of the 8-bit operators: what a call does besides its numbers."""
import ctypes

import pytest
import torch

import paper_1501_06633_b200 as mx
from paper_1501_06633_b200 import train8

pytestmark = pytest.mark.gpu
CALLS = ("quant8", "dequant8", "gemm8", "layer_norm_fprop", "layer_norm_bprop", "act8_fprop", "act8_bprop")


def test_other_threads_run_during_a_call():
    """The interpreter's lock is released around the library's call, as ctypes does: in the library's place
    stands the function that tells whether this thread holds it."""
    lib = train8._library()
    plain = train8._plain
    assert plain is not train8._NoPlain, "the marshalling module is not built"
    held = ctypes.cast(ctypes.pythonapi.PyGILState_Check, ctypes.c_void_p).value
    ours = [ctypes.cast(getattr(lib, "maxdnn_" + n), ctypes.c_void_p).value for n in CALLS]
    e8 = lambda *s: torch.zeros(*s, dtype=torch.uint8, device="cuda")
    f32 = lambda *s: torch.zeros(*s, device="cuda")
    q, s, x, v = e8(4, 128), e8(1, 4), f32(4, 128), f32(4)
    none = (None, None)
    f = mx.DTYPE_F32
    calls = {
        "quant8": (mx.Quant8Desc.make(4, 128, x_type=f), x, None, q, s, *none, *none, None),
        "dequant8": (mx.Quant8Desc.make(4, 128, x_type=f), 0, q, s, x, None),
        "gemm8": (mx.Gemm8Desc.make(4, 4, 128, c_type=f, b_block=mx.BLOCK_ROW), q, s, q, s, f32(4, 4), None),
        "layer_norm_fprop": (mx.LayerNormDesc.make(4, 128, x_type=f), x, None, None, x, v, v, *none, *none, None),
        "layer_norm_bprop": (mx.LayerNormDesc.make(4, 128, x_type=f), x, x, None, None, v, v, x, None, None, None, None),
        "act8_fprop": (mx.Act8Desc.make(4, 128, gated=False, x_type=f), x, x, *none, *none, None),
        "act8_bprop": (mx.Act8Desc.make(4, 128, gated=False, x_type=f), x, x, None, x, None),
    }
    try:
        plain.bind(*[held] * 7)
        got = {n: getattr(plain, n)(*calls[n]) for n in CALLS}
    finally:
        plain.bind(*ours)
    assert got == {n: 0 for n in CALLS}          # (1: held, -1: the call was not plain)
    mx.quant8(calls["quant8"][0], x, row=(q, s))
    assert bool((s == 127).all())


def test_both_ways_of_marshalling_make_the_same_calls(monkeypatch):
    """The example's forward and backward pass with the module, and with every call checked in Python."""
    import importlib.util
    import os
    at = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "feed_forward8.py")
    spec = importlib.util.spec_from_file_location("feed_forward8", at)
    ff = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ff)
    gen = torch.Generator(device="cuda").manual_seed(0)
    x, dout = (torch.randn(70, 200, device="cuda", generator=gen).to(torch.bfloat16) for _ in range(2))
    got = []
    for plain in (train8._library() and train8._plain, train8._NoPlain):
        monkeypatch.setattr(train8, "_plain", plain)
        block, before = ff.FeedForward8(200, 150, seed=1), mx.launch_count()
        got.append([block.forward(x), block.backward(dout), mx.launch_count() - before])
    (out, grads, n), (out2, grads2, n2) = got
    assert n == n2 and torch.equal(out, out2) and all(torch.equal(grads[k], grads2[k]) for k in grads)
