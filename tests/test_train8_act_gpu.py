"""Activations of fp32 values, in fp32.

Tolerance.  The functions that enter are within five units in the last place by CUDA's documented bounds
(exponential 2, normal distribution function 5, quotient up to 2), the products and sums around them add one
rounding each: 8 x 2^-23 = 2^-20 of each term of the result.  An exponential's argument z that was computed
brings its own error: at most six roundings (tanh form), 3 x 2^-23 z of the result; so does 1 - s in a
derivative, whose error is a rounding of s, times a factor of at most 3 z.  The derivatives are sums of two terms."""
import numpy as np
import pytest
import torch
from scipy import special

import paper_1501_06633_b200 as mx
from test_train8_gpu import ACTS, WIDE, as_held, down, within

pytestmark = pytest.mark.gpu


def cases():
    g = np.concatenate([np.linspace(-12, 12, 4001), -np.logspace(-8, 1, 600), np.logspace(-8, 1.6, 600), [0.0, -0.0]])
    return np.float32(g).astype(np.float64)


def terms(act, g):
    """f, and the two terms of f' (64 bits)."""
    if act == "silu":
        s, t = 1 / (1 + np.exp(-g)), 1 / (1 + np.exp(g))
        return g * s, s, g * s * t
    if act == "gelu":
        p = special.ndtr(g)              # (exact in the tail, where torch's function of this name is 0)
        return g * p, p, g * np.exp(-g * g / 2) / np.sqrt(2 * np.pi)
    k = 2 * np.sqrt(2 / np.pi)
    z = k * (g + 0.044715 * g ** 3)
    with np.errstate(over="ignore"):
        s, t = 1 / (1 + np.exp(-z)), 1 / (1 + np.exp(z))
    return g * s, s, g * s * t * k * (1 + 3 * 0.044715 * g * g)


@pytest.mark.parametrize("act", list(ACTS))
@pytest.mark.parametrize("gated", [False, True])
def test_fp32_activations_to_a_few_units(act, gated):
    g = cases()
    rng = np.random.default_rng(1)
    u = np.float32(rng.uniform(0.5, 2, g.size)).astype(np.float64)
    da = np.float32(rng.uniform(0.5, 2, g.size)).astype(np.float64)
    cols, many = g.size, 2 if gated else 1
    h = torch.from_numpy(np.concatenate([g, u]) if gated else g).float().cuda().view(1, many * cols)
    d = mx.Act8Desc.make(1, cols, act=ACTS[act], gated=gated, x_type=mx.DTYPE_F32)
    a, dh = torch.empty(1, cols, device="cuda"), torch.empty(1, many * cols, device="cuda")
    mx.act8_fprop(d, h, a=a)
    mx.act8_bprop(d, torch.from_numpy(da).float().cuda().view(1, cols), h, dh)
    f, t1, t2 = terms(act, g)
    uu = u if gated else 1.0
    z = np.abs(g) if act == "silu" else g * g / 2 if act == "gelu" else 2 * np.sqrt(2 / np.pi) * np.abs(g + 0.044715 * g ** 3)
    tol_d = 2.0 ** -20 + 3 * 2.0 ** -23 * z
    tol = tol_d if act == "gelu_tanh" else 2.0 ** -20
    tiny = 2.0 ** -126 * 8         # what falls below the normal numbers
    assert np.all(np.abs(down(a)[0] - f * uu) <= tol * np.abs(f * uu) + tiny)
    got = down(dh)[0]
    size = np.abs(t1) + np.abs(t2)
    assert np.all(np.abs(got[:cols] - da * uu * (t1 + t2)) <= tol_d * np.abs(da * uu) * size + tiny)
    if gated:
        assert np.all(np.abs(got[cols:] - da * f) <= tol * np.abs(da * f) + tiny)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_gelu_of_16_bit_values_far_below_zero(kind):
    """f = g P(g) where P is small: a few roundings of the exponential's argument (up to 72), 3 x 72 x 2^-24 of the
    value, and of its own growing error, 1.2 x 72 x 2^-23: 2^-15.  The result is rounded once."""
    g = as_held(-np.linspace(2.0, 12.0, 997), kind)
    n = g.size
    h = torch.from_numpy(np.concatenate([g, np.ones(n)])).to(WIDE[kind][1]).cuda().view(1, 2 * n)
    d = mx.Act8Desc.make(1, n, act=mx.ACT_GELU, x_type=WIDE[kind][0])
    a, dh = (torch.empty(1, m * n, dtype=WIDE[kind][1], device="cuda") for m in (1, 2))
    mx.act8_fprop(d, h, a=a)
    mx.act8_bprop(d, torch.ones(1, n, dtype=WIDE[kind][1], device="cuda"), h, dh)
    want = g * special.ndtr(g)
    for got in (down(a)[0], down(dh)[0, n:]):
        within(got, want, 2.0 ** -15 * np.abs(want), kind)
