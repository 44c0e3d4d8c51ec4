"""Gradients of log probabilities from infinite gradients of the results: an infinity with the sign of the formula where p is
not 0, in its row alone, in every form of the result.  A block's scale is that of its finite values."""
import numpy as np
import pytest
import torch

import paper_1501_06633_b200 as mx
import train8_ref as ref
from test_train8_gpu import PACKED, WIDE, bytes_of, down

pytestmark = pytest.mark.gpu


def given(rows, cols, kind, seed=0):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.uniform(-4, 4, (rows, cols))).to(WIDE[kind][1]).cuda()
    target = torch.from_numpy(rng.integers(0, cols, rows)).cuda()
    dlp = torch.from_numpy(rng.standard_normal(rows)).float().cuda()
    return x, target, dlp, torch.logsumexp(x.double(), 1).float()


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_wide(kind):
    rows, cols = 5, 1003
    x, target, dlp, lse = given(rows, cols, kind)
    dlp[1], dlp[3] = float("inf"), -float("inf")
    dx = torch.empty_like(x)
    mx.logprob_bprop(mx.LogprobDesc.make(rows, cols, x_type=WIDE[kind][0]), x, target, lse, dlogprob=dlp, dx=dx)
    got, n = down(dx), np.arange(cols)
    for r, sign in ((1, 1), (3, -1)):
        np.testing.assert_array_equal(got[r], np.where(n == int(target[r]), sign, -sign) * np.inf)
    assert np.isfinite(got[[0, 2, 4]]).all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("packed", ["e4m3", "e5m2"])
@pytest.mark.parametrize("rows,cols", [(130, 264), (129, 301)])
def test_packed(kind, packed, rows, cols):
    """E5M2 holds the infinities, E4M3 has none and holds NaN; the other rows' values and all scales are as if the infinite rows'
    values were not there."""
    x, target, dlp, lse = given(rows, cols, kind, 3)
    t = PACKED[packed][0]
    d = mx.LogprobDesc.make(rows, cols, x_type=WIDE[kind][0], q_type=t)

    def call(dlp):
        row = (mx.empty_packed(rows, cols, t), mx.empty_scales(mx.BLOCK_ROW, rows, cols))
        col = (mx.empty_packed(rows, cols, t), mx.empty_scales(mx.BLOCK_COL, rows, cols))
        mx.logprob_bprop(d, x, target, lse, dlogprob=dlp, row=row, col=col)
        return [down(row[0]), bytes_of(row[1]), down(col[0]), bytes_of(col[1])]

    bad, calm = dlp.clone(), dlp.clone()
    at = [1, 100, rows - 1]
    bad[at], calm[at] = float("inf"), 0.0
    got, want = call(bad), call(calm)
    others = np.setdiff1d(np.arange(rows), at)
    for q, w in ((got[0], want[0]), (got[2], want[2])):
        np.testing.assert_array_equal(q[others], w[others])
        for r in at:
            sign = np.where(np.arange(cols) == int(target[r]), 1, -1)
            if packed == "e5m2":
                np.testing.assert_array_equal(q[r], sign * np.inf)
            else:
                assert np.isnan(q[r]).all()
    np.testing.assert_array_equal(got[3], want[3])
    np.testing.assert_array_equal(got[1][:, others], want[1][:, others])
    assert np.all(ref.value_of(got[1][:, at]) == 1.0)           # no finite value: as a block of zeros


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_infinite_gradients_of_the_entropy_and_masked_logits(kind):
    """An infinite dentropy gives infinities or NaN throughout its row, an infinite dlogprob NaN where p is 0; no other row is touched."""
    rows, cols = 4, 300
    x, target, dlp, lse = given(rows, cols, kind, 5)
    x[:, 7], x[:, 250:] = -float("inf"), -float("inf")
    target %= 7
    lse = torch.logsumexp(x.double(), 1).float()
    entropy = torch.distributions.Categorical(logits=x.float()).probs
    entropy = -torch.special.xlogy(entropy, entropy).sum(1)
    dh = torch.ones(rows, device="cuda")
    dlp[1], dh[2] = float("inf"), -float("inf")
    dx = torch.empty_like(x)
    mx.logprob_bprop(mx.LogprobDesc.make(rows, cols, x_type=WIDE[kind][0]), x, target, lse, dlogprob=dlp, entropy=entropy, dentropy=dh, dx=dx)
    got, masked = down(dx), np.isinf(down(x)[0])
    assert np.isfinite(got[[0, 3]]).all() and np.all(got[[0, 3]][:, masked] == 0) and not np.isfinite(got[2]).any()
    np.testing.assert_array_equal(np.isnan(got[1]), masked)
    np.testing.assert_array_equal(got[1][~masked], np.where(np.arange(cols) == int(target[1]), 1, -1)[~masked] * np.inf)
