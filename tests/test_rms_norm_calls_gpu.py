"""RMS norm: workspaces that are refused (planned for the device, so not without one), and results in their inputs' memory."""
import ctypes

import pytest
import torch

import paper_1501_06633_b200 as mx
from paper_1501_06633_b200 import train8
from test_train8_gpu import WIDE

pytestmark = pytest.mark.gpu


def test_workspaces_that_are_refused():
    rows, cols = 40, 264
    d = mx.RmsNormDesc.make(rows, cols, x_type=mx.DTYPE_F32)
    h, dy = (torch.randn(rows, cols, device="cuda") for _ in range(2))
    dx, rstd, dg = torch.full((rows, cols), 7.0, device="cuda"), torch.ones(rows, device="cuda"), torch.full((cols,), 7.0, device="cuda")
    need = mx.rms_norm_bprop_workspace(d)
    ws = torch.empty(need + 16, dtype=torch.uint8, device="cuda")

    def call(dgamma, at, size):
        return train8._library().maxdnn_rms_norm_bprop(ctypes.byref(d), dy.data_ptr(), h.data_ptr(), None, None, rstd.data_ptr(), None, dx.data_ptr(),
                                                       dgamma, at, size, torch.cuda.current_stream().cuda_stream)

    for at, size in ((None, need), (ws.data_ptr() + 4, need), (ws.data_ptr(), 0), (ws.data_ptr(), need - 1)):
        assert call(dg.data_ptr(), at, size) == mx.INVALID_VALUE
    torch.cuda.synchronize()
    assert bool((dg == 7).all()) and bool((dx == 7).all())          # nothing was launched
    assert call(dg.data_ptr(), ws.data_ptr(), need) == mx.OK
    want, wg = dx.clone(), dg.clone()
    dx.fill_(7.0)
    assert call(None, None, 0) == mx.OK                               # no sums, no workspace
    torch.cuda.synchronize()
    assert torch.equal(dx, want) and bool((wg != 7).all())


@pytest.mark.parametrize("rows,cols,pad", [(5, 11, 0), (3700, 13, 0), (3700, 12, 1), (3700, 521, 2), (905, 2051, 1), (300, 4101, 0), (900, 4096, 0), (3, 20001, 1)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_results_in_their_inputs_memory(rows, cols, pad, kind):
    """The sum in x's place, with a residual and without; dx in dy's: the same bits as in memory of their own."""
    code, tt = WIDE[kind]
    ld = cols + pad
    gen = torch.Generator(device="cuda").manual_seed(cols)
    x, r, dy = (torch.randn(rows, ld, device="cuda", generator=gen).to(tt) for _ in range(3))
    d = mx.RmsNormDesc.make(rows, cols, x_type=code, ldx=ld, ldr=ld, ldy=ld)
    for residual in (r[:, :cols], None):
        s, y, y2, rstd, rstd2 = *(torch.full((rows, ld), 7.0, dtype=tt, device="cuda") for _ in range(3)), *(torch.empty(rows, device="cuda") for _ in range(2))
        mx.rms_norm_fprop(d, x[:, :cols], residual=residual, sum=s[:, :cols], y=y[:, :cols], rstd=rstd)
        into = x.clone()
        mx.rms_norm_fprop(d, into[:, :cols], residual=residual, sum=into[:, :cols], y=y2[:, :cols], rstd=rstd2)
        assert torch.equal(into[:, :cols], s[:, :cols]) and torch.equal(into[:, cols:], x[:, cols:])
        assert torch.equal(y2, y) and torch.equal(rstd2, rstd)
    dx, dg, dg2 = torch.full((rows, ld), 7.0, dtype=tt, device="cuda"), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ws = torch.empty(mx.rms_norm_bprop_workspace(d), dtype=torch.uint8, device="cuda")
    mx.rms_norm_bprop(d, dy[:, :cols], s[:, :cols], None, rstd, dx[:, :cols], dg, ws)
    into = dy.clone()
    mx.rms_norm_bprop(d, into[:, :cols], s[:, :cols], None, rstd, into[:, :cols], dg2, ws)
    assert torch.equal(into[:, :cols], dx[:, :cols]) and torch.equal(into[:, cols:], dy[:, cols:]) and torch.equal(dg, dg2)
    assert mx.last_device_status() == mx.OK
