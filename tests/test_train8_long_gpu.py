"""Long reductions of terms of one sign whose sums do not fit 24 bits, which is where a truncating accumulator
drifts.

Tolerance.  A running sum of n matrix instructions (32 terms each) loses at most two units in its last place,
2^-22 of it, at each: one where the terms are aligned, one where they are added.  With terms of one
size the running sum grows evenly, so that is at most 2^-22 (n + 1) / 2 of the final sum; partial sums of
c accumulators are added with at most 2^-24 (c + 1) / 2.  An accumulator holds 16 blocks (n = 64) of an fp32 result,
128 (n = 512) of a 16-bit one.  One accumulator for the whole reduction would lose about 2.1e-8 (half a unit, at a
mean of 0.7 of 2^-23) per instruction: 4.3e-5 over 65536 terms, 6.9e-4 over 2^20, against bounds of 8.7e-6 and 6.4e-5."""
import pytest
import torch

import paper_1501_06633_b200 as mx

pytestmark = pytest.mark.gpu

TYPES = {"f32": (mx.DTYPE_F32, torch.float32, 16), "f16": (mx.DTYPE_F16, torch.float16, 128), "bf16": (mx.DTYPE_BF16, torch.bfloat16, 128)}


def operand(rows, K, gen):
    """E4M3 numbers from 1 to 1.875 with any mantissa, a scale of 2^-11 to 2^-9 per row and block: (values, scales)."""
    q = torch.randint(0x38, 0x40, (rows, K), dtype=torch.uint8, device="cuda", generator=gen)
    s = torch.randint(127 - 11, 127 - 8, (K // 128, rows), dtype=torch.uint8, device="cuda", generator=gen)
    return q, s


def exact(a, b, K):
    """The product in 64 bits, 8192 terms at a time."""
    total = 0
    for k in range(0, K, 8192):
        part = []
        for q, s in (a, b):
            v = q[:, k:k + 8192].view(torch.float8_e4m3fn).to(torch.float32).double()
            e = s[k // 128:(k + 8192) // 128].to(torch.int32) - 127
            part.append(v * torch.pow(2.0, e.double()).t().repeat_interleave(128, 1))
        total = total + part[0] @ part[1].t()
    return total


@pytest.mark.parametrize("ct,K", [("f32", 16384), ("f32", 65536), ("f16", 1 << 20), ("bf16", 1 << 18)])
@pytest.mark.parametrize("pair,cols", [(-1, 16), (-1, 128), (1, 128), (1, 224), (1, 256)])
def test_sums_of_one_sign(ct, K, pair, cols):
    code, dtype, blocks = TYPES[ct]
    gen = torch.Generator(device="cuda").manual_seed(K + cols)
    M, N = (256, 256) if pair > 0 else (128, 128)
    a, b = operand(M, K, gen), operand(N, K, gen)
    c = torch.empty(M, N, dtype=dtype, device="cuda")
    mx.set_option("GEMM8_PAIR", pair)
    mx.set_option("GEMM8_COLS", cols)
    mx.set_option("GEMM8_SPLIT", 1)
    d = mx.Gemm8Desc.make(M, N, K, c_type=code, b_block=mx.BLOCK_ROW)
    mx.gemm8(d, a[0], a[1], b[0], b[1], c)
    assert mx.last_device_status() == mx.OK
    want = exact(a, b, K)
    n, parts = 4 * blocks, -(-K // (128 * blocks))
    tol = (2.0 ** -22 * (n + 1) / 2 + 2.0 ** -24 * (parts + 1) / 2) * want
    # rounding keeps order: the result lies between the interval's rounded ends
    assert bool((c >= (want - tol).to(dtype)).all()) and bool((c <= (want + tol).to(dtype)).all())
