"""A bounded wait that runs out in either kernel of the orthogonalised update: the call ends, its status says so, and the next call
is what it was (an arrival that never comes stands in for the failure)."""
import pytest
import torch

import paper_1501_06633_b200 as mx
from test_orthogonalise_gpu import call, gradients

pytestmark = pytest.mark.gpu


# one CTA, several matrices of two, sixteen; through memory
@pytest.mark.parametrize("batch,rows,cols", [(1, 16, 16), (4, 128, 512), (1, 3000, 100), (1, 300, 140)])
def test_a_wait_that_runs_out_is_reported(batch, rows, cols):
    x = gradients(batch, rows, cols, "bf16", 40)
    want = call(x, "bf16")
    d = mx.OrthoDesc.make(rows, cols, batch=batch)
    out, ws = torch.empty_like(want), torch.empty(mx.orthogonalise_workspace(d), dtype=torch.uint8, device="cuda")
    mx.set_option("TEST_MISSING_ARRIVAL", 1)
    try:
        mx.orthogonalise(d, x, out, ws)
    finally:
        mx.reset_options()
    assert mx.last_device_status() == mx.DEVICE_TIMEOUT
    assert torch.equal(call(x, "bf16"), want)
