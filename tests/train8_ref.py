"""Plain definitions of the 8-bit training operators in 64 bits (numpy / torch CPU), for the tests.
Shares no code with the library or its binding."""
import numpy as np
import torch

BLOCK = 128
SPEC = {"e4m3": (448.0, 3, -6, torch.float8_e4m3fn), "e5m2": (57344.0, 2, -14, torch.float8_e5m2)}


def blocks(n):
    return -(-n // BLOCK)


def cells(form, rows, cols):
    """(scale index along the storage layout, rows slice, cols slice) of each block."""
    br, bc = {"row": (1, BLOCK), "col": (BLOCK, 1), "tile": (BLOCK, BLOCK)}[form]
    for r in range(0, rows, br):
        for c in range(0, cols, bc):
            at = (c // BLOCK, r) if form == "row" else (r // BLOCK, c // bc)
            yield at, slice(r, min(r + br, rows)), slice(c, min(c + bc, cols))


def scale_shape(form, rows, cols):
    return {"row": (blocks(cols), rows), "col": (blocks(rows), cols), "tile": (blocks(rows), blocks(cols))}[form]


def pack(x, form, kind):
    """(values that q holds, scale bytes) of a float64 matrix; NaN where the result is NaN."""
    top, bits, least, _ = SPEC[kind]
    q, s = np.zeros_like(x), np.zeros(scale_shape(form, *x.shape), np.uint8)
    for at, rs, cs in cells(form, *x.shape):
        v = x[rs, cs]
        m = np.max(np.where(np.isfinite(v), np.abs(v), 0.0))
        e = 0
        if m > 0:
            e = int(np.floor(np.log2(m / top))) - 2
            while top * 2.0 ** e < m:
                e += 1
            e = min(max(e, -126), 127)
        s[at] = e + 127
        w = v / 2.0 ** e
        fin = np.isfinite(w)
        _, ex = np.frexp(np.where(fin, w, 0.0))
        step = 2.0 ** (np.maximum(ex - 1, least) - bits)
        r = np.round(np.where(fin, w, 0.0) / step) * step
        bad = np.full_like(w, np.nan) if kind == "e4m3" else w
        q[rs, cs] = np.where(fin, r, bad)
    return q, s


def value_of(byte):
    b = byte.astype(np.float64)
    return np.where(byte == 255, np.nan, 2.0 ** (b - 127))


def spread(scale, form, rows, cols):
    """The scale of each value, as a [rows][cols] matrix, from numbers in the storage layout."""
    out = np.zeros((rows, cols))
    for at, rs, cs in cells(form, rows, cols):
        out[rs, cs] = scale[at]
    return out


def normal_cdf(g):
    return torch.special.ndtr(torch.from_numpy(g)).numpy()


def act(kind, g):
    """f(g) and f'(g)."""
    with np.errstate(over="ignore"):
        if kind == "silu":
            s = 1 / (1 + np.exp(-g))
            return g * s, s * (1 + g * (1 - s))
        if kind == "gelu":
            p = normal_cdf(g)
            return g * p, p + g * np.exp(-g * g / 2) / np.sqrt(2 * np.pi)
        k = np.sqrt(2 / np.pi)
        t = np.tanh(k * (g + 0.044715 * g ** 3))
        return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g)


def layer_norm(x, gamma, beta, eps):
    mean = x.mean(1, keepdims=True)
    rstd = 1 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    return (x - mean) * rstd * gamma + beta, mean[:, 0], rstd[:, 0]


def layer_norm_grads(x, dy, gamma, mean, rstd):
    xh = (x - mean[:, None]) * rstd[:, None]
    g = dy * gamma
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    return dx, (dy * xh).sum(0), dy.sum(0)
