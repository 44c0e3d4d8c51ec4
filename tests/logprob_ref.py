"""Plain definitions of the log probabilities and their gradient in 64 bits (numpy), for the tests."""
import numpy as np


def forward(x, scale, target, top):
    """lse, logprob, entropy, (values, indices) of the largest, and the mean and mean square distance to the maximum under p."""
    rows, cols = x.shape
    z = x * scale
    with np.errstate(invalid="ignore", divide="ignore"):
        m = z.max(1, keepdims=True)
        nothing = m[:, 0] == -np.inf
        far = np.where(nothing[:, None], -np.inf, z - m)
        e = np.exp(far)
        total = e.sum(1)
        ln = np.log(total)
        p = np.where(nothing[:, None], 0.0, e / total[:, None])
        far0 = np.where(e > 0, far, 0.0)
        a1, a2 = (p * -far0).sum(1), (p * far0 ** 2).sum(1)
        lse = np.where(nothing, -np.inf, m[:, 0] + ln)
        entropy = np.where(nothing, 0.0, ln + a1)
    token = (target >= 0) & (target < cols)
    at = np.where(token, target, 0)
    with np.errstate(invalid="ignore"):
        lp = np.where(nothing, -np.inf, z[np.arange(rows), at] - m[:, 0] - ln)
    lp = np.where(token, lp, 0.0)
    idx = np.argsort(-x, axis=1, kind="stable")[:, :top]
    idx = np.pad(idx, ((0, 0), (0, top - idx.shape[1])))
    v = np.take_along_axis(x, idx, 1)
    v[:, cols:] = -np.inf
    with np.errstate(invalid="ignore"):
        tlp = np.where(v == -np.inf, -np.inf, v * scale - m - ln[:, None])
    return lse, lp, entropy, tlp, np.where(v == -np.inf, -1, idx), a1, a2


def gradient(x, scale, target, lse, dlp, entropy, dh):
    """dx and the size of the terms it is made of."""
    rows, cols = x.shape
    token = (target >= 0) & (target < cols)
    nothing = lse == -np.inf
    dlp = np.where(token & ~nothing, dlp, 0.0)
    with np.errstate(invalid="ignore"):
        l = np.where(nothing[:, None] | (x == -np.inf), -np.inf, x * scale - lse[:, None])
    p = np.exp(l)
    l0 = np.where(p > 0, l, 0.0)
    dx = -p * dlp[:, None] - dh[:, None] * p * (l0 + entropy[:, None])
    rel = 2.0 ** -21 + np.abs(l0) * 2.0 ** -22
    size = scale * p * (np.abs(dlp)[:, None] + np.abs(dh)[:, None] * (np.abs(l0) + np.abs(entropy)[:, None]))
    dx[np.arange(rows), np.where(token, target, 0)] += dlp
    return dx * scale, rel * size + 2.0 ** -23 * np.abs(dx * scale) + 1e-36 * (1 + size.max())
