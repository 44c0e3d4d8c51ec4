"""Small matrices of the orthogonalised update where a cluster for them cannot be had (here: may not): they go through memory.
Tolerances: see test_orthogonalise_gpu.py."""
import pytest
import torch

import paper_1501_06633_b200 as mx
from test_orthogonalise_gpu import call, formula, gradients, near

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 1), (1, 1, 9), (2, 5, 3), (1, 16, 16), (3, 32, 100), (4, 128, 512), (1, 127, 129),
                                             (2, 90, 1000), (1, 2000, 100), (1, 100, 4000)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_small_matrices_through_memory(batch, rows, cols, kind):
    x = gradients(batch, rows, cols, kind, rows)
    parts = -(-max(rows, cols) // 256)
    want = formula(x, 5)
    try:
        for most in {0, 1, 8, parts}:
            mx.set_option("ORTHO_CLUSTER", most)
            before = mx.launch_count()
            near(call(x, kind), want)
            assert mx.launch_count() - before == (1 if parts <= most else 3)      # (the sum of squares, X, all steps)
    finally:
        mx.reset_options()
    before = mx.launch_count()
    kept = call(x, kind)
    assert mx.launch_count() - before == 1
    near(kept, want)
    assert mx.last_device_status() == mx.OK
