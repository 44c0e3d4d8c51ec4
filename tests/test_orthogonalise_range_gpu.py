"""The orthogonalised update's special values and sizes of gradients through both of its kernels: matrices that a cluster keeps
(shorter side up to 128, longer up to 4096), alone in a CTA and shared by 2 to 16, and those that go through memory.
Tolerances: see test_orthogonalise_gpu.py."""
import pytest
import torch

import paper_1501_06633_b200 as mx
from test_orthogonalise_gpu import call, formula, gradients, near

pytestmark = pytest.mark.gpu
KEPT = [(16, 16), (64, 100), (128, 128), (400, 60), (90, 1000), (2000, 100), (100, 4000)]
CHAIN = [(130, 260), (300, 140)]


@pytest.mark.parametrize("rows,cols", KEPT + CHAIN)
@pytest.mark.parametrize("size", [1e-35, 1e-30, 1e-20, 1e-18, 1e-17, 1e-16, 1e-14, 1e-10, 1e-8, 1e-7, 1e-6, 1e-4, 1e20, 1e35])
def test_any_size_of_gradient(rows, cols, size):
    """|G| far below eps, around it and far above, in few and many steps: as close to the formula everywhere."""
    x = gradients(1, rows, cols, "f32", rows).double()
    x = (x / x.norm() * size).float()
    for steps in (5, 1, 6):
        want = formula(x, steps)
        near(call(x, "f32", steps), want)


@pytest.mark.parametrize("rows,cols", KEPT + CHAIN)
def test_steps_that_shrink(rows, cols):
    """Coefficients below 1 make X smaller from step to step."""
    x = gradients(1, rows, cols, "f32", 2)
    near(call(x, "f32", 5, (0.1, -0.05, 0.0)), formula(x, 5, [(0.1, -0.05, 0.0)] * 5))


@pytest.mark.parametrize("rows,cols", KEPT + CHAIN)
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("top", [1.5e38, 2e38, 3.2e38, 3.38e38])
def test_entries_near_the_largest_number(rows, cols, kind, top):
    """Finite entries count, whatever their exponent: alone, next to ordinary ones, and throughout."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    for which in ("one", "some", "all"):
        if which == "all":
            x = torch.rand(1, rows, cols, device="cuda", generator=gen).sub_(0.5).sign_().mul_(top)
            x[0, :, ::3] *= 0.9
        else:
            x = torch.randn(1, rows, cols, device="cuda", generator=gen)
            x[0, rows // 2, cols // 2] = top
            if which == "some":
                x[0, 0, :] = -top
                x[0, 1, ::2] = 0.25 * top
        x = x.to(torch.float32 if kind == "f32" else torch.bfloat16)
        near(call(x, kind), formula(x, 5))


@pytest.mark.parametrize("rows,cols", KEPT + CHAIN)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_zeros_and_values_that_are_not_finite(rows, cols, kind):
    x = gradients(6, rows, cols, kind, 5)
    x[1] = 0
    x[2, 3, 5] = float("nan")
    x[3, rows - 1, cols - 1] = float("inf")
    x[4, 0, 0] = -float("inf")
    d = mx.OrthoDesc.make(rows, cols, batch=6)
    # a workspace that holds NaN before the call
    ws = torch.full((mx.orthogonalise_workspace(d) // 2,), float("nan"), dtype=torch.float16, device="cuda").view(torch.uint8)
    got = call(x, kind, ws=ws)
    assert bool((got[1] == 0).all()) and all(bool(torch.isnan(got[i]).all()) for i in (2, 3, 4))
    for i in (0, 5):
        near(got[i:i + 1], formula(x[i:i + 1], 5))
