"""The orthogonalised update against its definition in 64 bits.

Tolerance.  X is held in 22 bits, the products' operands in FP16 (half a step 2^-12 of an entry, up to the residues of the
diagonals): a step adds at most about 4 x 2^-12 of the result's norm in the directions that it keeps (the products' operands X, A,
B and X again), which a later step multiplies by |p'| <= 1.6 where a singular value is near 1 and leaves alone (relative to
the value) where it is small: 5 steps, 20 x 2^-12 = 2^-7.6 at the most, as independent roundings sqrt(20) x 2^-12 / sqrt(3) = 6e-4 of its
norm.  Held here to 2^-9 = 2e-3 of the norm, with the rounding to BF16 besides: half a step is up to 2^-8 of an entry (the value
just above a power of two), so at most 2^-8 of the norm; as roundings of many entries, spread evenly over their half steps, at most
2^-8 / sqrt(3).  A single entry: 12 times the root mean square of that."""
import numpy as np
import pytest
import torch

import paper_1501_06633_b200 as mx

pytestmark = pytest.mark.gpu
DEFAULT = (3.4445, -4.7750, 2.0315)
TYPES = {"f32": (mx.DTYPE_F32, torch.float32), "bf16": (mx.DTYPE_BF16, torch.bfloat16), "f16": (mx.DTYPE_F16, torch.float16)}
def share(entries):
    return 2.0 ** -9 + 2.0 ** -8 / (3 ** 0.5 if entries >= 64 else 1)


def formula(x, steps, coefficients=None, eps=1e-7):
    """[batch][rows][cols] in 64 bits."""
    x = x.double()
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2) if tall else x
    x = x / (x.flatten(1).norm(dim=1)[:, None, None] + eps)
    for i in range(steps):
        a, b, c = (coefficients or [DEFAULT] * steps)[i]
        gram = x @ x.transpose(1, 2)
        x = a * x + (b * gram + c * gram @ gram) @ x
    return x.transpose(1, 2) if tall else x


def gradients(batch, rows, cols, kind, seed, spectrum="mixed"):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    new = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    if spectrum == "mixed":
        k = max(1, min(rows, cols) // 16)
        x = torch.bmm(new(batch, rows, k), new(batch, k, cols)) / k ** 0.5 + 0.1 * new(batch, rows, cols)
    else:
        x = new(batch, rows, cols)
    return (1e-3 * x).to(TYPES[kind][1])


def call(x, kind, steps=5, coefficients=None, out=None, ws=None, **pitches):
    batch, rows, cols = x.shape
    d = mx.OrthoDesc.make(rows, cols, batch=batch, steps=steps, x_type=TYPES[kind][0], **pitches)
    out = torch.empty(batch, rows, cols, dtype=torch.bfloat16, device="cuda") if out is None else out
    ws = torch.empty(mx.orthogonalise_workspace(d), dtype=torch.uint8, device="cuda") if ws is None else ws
    mx.orthogonalise(d, x, out, ws, coefficients)
    assert mx.last_device_status() == mx.OK
    return out


def near(got, want):
    for g, w in zip(got.double(), want):
        rms, part = float(w.norm()) / w.numel() ** 0.5, share(w.numel())
        assert float((g - w).norm()) <= part * float(w.norm()), float((g - w).norm()) / float(w.norm())
        assert float((g - w).abs().max()) <= 12 * part * max(rms, float(w.abs().max()) / 12)


# every tile shape, sizes that end inside tiles, stages and vectors of eight, taller and wider
@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 1), (1, 1, 9), (2, 5, 3), (1, 16, 16), (3, 32, 100), (2, 100, 31), (1, 64, 64), (1, 127, 129),
                                             (1, 128, 128), (4, 128, 512), (2, 200, 130), (1, 129, 1000), (1, 1000, 129), (1, 256, 256),
                                             (1, 300, 700), (1, 520, 264), (1, 777, 777), (1, 1024, 1024), (1, 1000, 2309), (1, 2309, 1000),
                                             (40, 256, 128), (9, 264, 520), (1, 2048, 2048), (1, 4096, 1000)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_against_the_formula(batch, rows, cols, kind):
    x = gradients(batch, rows, cols, kind, rows + cols)
    near(call(x, kind), formula(x, 5))
    if kind == "bf16":
        x = gradients(batch, rows, cols, kind, 7, "even")
        near(call(x, kind), formula(x, 5))


@pytest.mark.parametrize("steps", [1, 2, 3, 6])
@pytest.mark.parametrize("rows,cols", [(96, 200), (300, 140)])
def test_steps_with_coefficients_of_their_own(steps, rows, cols):
    x = gradients(2, rows, cols, "f32", steps)
    each = [(3.4445 - 0.2 * i, -4.7750 + 0.3 * i, 2.0315 - 0.1 * i) for i in range(steps)]
    near(call(x, "f32", steps, each), formula(x, steps, each))
    near(call(x, "f32", steps, (1.5, -0.5, 0.0)), formula(x, steps, [(1.5, -0.5, 0.0)] * steps))
    assert torch.equal(call(x, "f32", steps), call(x, "f32", steps, DEFAULT))


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols,pad,pado", [(100, 200, 8, 8), (100, 200, 3, 5), (201, 99, 0, 1), (64, 64, 7, 0)])
def test_pitches_leave_their_gaps_alone(kind, rows, cols, pad, pado):
    x = gradients(2, rows, cols, kind, 3)
    wide = torch.full((2, rows + 1, cols + pad), float("nan"), dtype=x.dtype, device="cuda")
    wide[:, :rows, :cols] = x
    out = torch.full((2, rows + 2, cols + pado), 7.0, dtype=torch.bfloat16, device="cuda")
    call(wide[:, :rows, :cols], kind, out=out[:, :rows, :cols], ldx=cols + pad, ldo=cols + pado, stride_x=(rows + 1) * (cols + pad),
         stride_o=(rows + 2) * (cols + pado))
    assert torch.equal(out[:, :rows, :cols], call(x, kind))
    assert bool((out[:, rows:] == 7).all()) and bool((out[:, :, cols:] == 7).all())
    one = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")
    d = mx.OrthoDesc.make(rows, cols, x_type=TYPES[kind][0])
    mx.orthogonalise(d, x[0].contiguous(), one, torch.empty(mx.orthogonalise_workspace(d), dtype=torch.uint8, device="cuda"))
    near(one[None], formula(x[:1], 5))


@pytest.mark.parametrize("size", [1e-30, 1e-20, 1.0, 1e18, 1e30])
def test_any_size_of_gradient(size):
    """The norm's square would leave the range of 32 bits."""
    x = gradients(1, 130, 260, "f32", 4) * 1e3
    got = call(x * size, "f32")
    near(got, formula((x * size), 5, eps=1e-7))


def test_zeros_and_values_that_are_not_finite():
    """In a batch, a matrix of zeros gives zeros and one with a NaN or infinity NaN; their neighbours are what they are alone."""
    x = gradients(5, 70, 150, "bf16", 5)
    x[1] = 0
    x[2, 3, 5] = float("nan")
    x[3, 69, 149] = float("inf")
    # a workspace that holds NaN before the call
    d = mx.OrthoDesc.make(70, 150, batch=5)
    ws = torch.full((mx.orthogonalise_workspace(d) // 2,), float("nan"), dtype=torch.float16, device="cuda").view(torch.uint8)
    got = call(x, "bf16", ws=ws)
    assert bool((got[1] == 0).all()) and bool(torch.isnan(got[2]).all()) and bool(torch.isnan(got[3]).all())
    for i in (0, 4):
        near(got[i:i + 1], formula(x[i:i + 1], 5))


def test_repeated_and_on_another_stream():
    """The same bits again, with workspaces of other contents, from another stream and from a graph."""
    for batch, rows, cols in ((1, 700, 1100), (6, 256, 64)):
        x = gradients(batch, rows, cols, "bf16", 8)
        want = call(x, "bf16")
        d = mx.OrthoDesc.make(rows, cols, batch=batch)
        ws = torch.randint(0, 255, (mx.orthogonalise_workspace(d),), dtype=torch.uint8, device="cuda")
        out = torch.zeros_like(want)
        other = torch.cuda.Stream()
        other.wait_stream(torch.cuda.current_stream())
        mx.orthogonalise(d, x, out, ws, stream=other)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            mx.orthogonalise(d, x, out, ws)
        for k in range(3):
            out.zero_()
            y = gradients(batch, rows, cols, "bf16", 20 + k)
            x.copy_(y)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, call(y, "bf16"))
        assert mx.last_device_status() == mx.OK


def test_two_calls_at_once():
    """Each call's CTAs wait for one another: two of them, and a product, on streams of their own."""
    xs = [gradients(1, 900, 1300, "bf16", 30), gradients(3, 400, 300, "bf16", 31)]
    want = [call(x, "bf16") for x in xs]
    outs = [torch.zeros_like(w) for w in want]
    ds = [mx.OrthoDesc.make(x.shape[1], x.shape[2], batch=x.shape[0]) for x in xs]
    wss = [torch.empty(mx.orthogonalise_workspace(d), dtype=torch.uint8, device="cuda") for d in ds]
    q, s = mx.empty_packed(2048, 2048), mx.empty_scales(mx.BLOCK_ROW, 2048, 2048)
    mx.quant8(mx.Quant8Desc.make(2048, 2048), torch.randn(2048, 2048, device="cuda").to(torch.bfloat16), row=(q, s))
    g = mx.Gemm8Desc.make(2048, 2048, 2048, b_block=mx.BLOCK_ROW)
    c, wc = (torch.zeros(2048, 2048, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mx.gemm8(g, q, s, q, s, wc)
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(10):
        for d, x, out, ws, st in zip(ds, xs, outs, wss, streams):
            mx.orthogonalise(d, x, out, ws, stream=st)
        mx.gemm8(g, q, s, q, s, c, stream=streams[2])
    torch.cuda.synchronize()
    assert mx.last_device_status() == mx.OK
    assert all(torch.equal(o, w) for o, w in zip(outs, want)) and torch.equal(c, wc)


def test_a_wait_that_runs_out_is_reported():
    x = gradients(1, 300, 300, "bf16", 40)
    want = call(x, "bf16")
    d = mx.OrthoDesc.make(300, 300)
    out, ws = torch.empty_like(want), torch.empty(mx.orthogonalise_workspace(d), dtype=torch.uint8, device="cuda")
    mx.set_option("TEST_MISSING_ARRIVAL", 1)
    mx.orthogonalise(d, x, out, ws)
    mx.reset_options()
    assert mx.last_device_status() == mx.DEVICE_TIMEOUT
    assert torch.equal(call(x, "bf16"), want)
