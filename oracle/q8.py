"""Oracle of the layer norm, the matrices in 8 bits with a scale for each block
of 128, their products, and the backward passes (float64 NumPy)."""
import numpy as np

from .kv8 import E_MAX, E_MIN, e4m3_numbers

BLOCK = 128


def layer_norm(x, w, b, cu, plus_one, eps):
    """(y, stats [rows][2] = mean, 1/sqrt(var + eps)); w, b [segments][cols] or None."""
    x = np.asarray(x, np.float64)
    mean = x.mean(axis=1, keepdims=True)
    rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(axis=1, keepdims=True) + eps)
    y = (x - mean) * rstd
    for i in range(len(cu) - 1):
        r = slice(int(cu[i]), int(cu[i + 1]))
        if w is not None:
            y[r] *= np.asarray(w[i], np.float64) + (1.0 if plus_one else 0.0)
        if b is not None:
            y[r] += np.asarray(b[i], np.float64)
    return y, np.concatenate([mean, rstd], axis=1)


def layer_norm_backward(x, stats, w, cu, plus_one, dy):
    """(dx, dw, db) by the chain rule, with the given mean and rstd."""
    x, dy, stats = (np.asarray(t, np.float64) for t in (x, dy, stats))
    xh = (x - stats[:, :1]) * stats[:, 1:]
    g = dy.copy()
    dw, db = np.zeros((len(cu) - 1, x.shape[1])), np.zeros((len(cu) - 1, x.shape[1]))
    for i in range(len(cu) - 1):
        r = slice(int(cu[i]), int(cu[i + 1]))
        if w is not None:
            g[r] *= np.asarray(w[i], np.float64) + (1.0 if plus_one else 0.0)
        dw[i], db[i] = (dy[r] * xh[r]).sum(axis=0), dy[r].sum(axis=0)
    dx = stats[:, 1:] * (g - g.mean(axis=1, keepdims=True) - xh * (g * xh).mean(axis=1, keepdims=True))
    return dx, dw, db


def exponents(x, square=False):
    """The exponent of every number's group, [rows][cols]."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    high = BLOCK if square else 1
    top = np.zeros((-(-rows // high) * high, -(-cols // BLOCK) * BLOCK))
    top[:rows, :cols] = np.abs(np.where(np.isfinite(x), x, 0.0))
    top = top.reshape(top.shape[0] // high, high, -1, BLOCK).max(axis=(1, 3))
    m, p = np.frexp(top / 448.0)  # top = 448 m 2^p, m in [0.5, 1)
    e = np.clip(np.where(top == 0.0, E_MIN, np.where(m == 0.5, p - 1, p)), E_MIN, E_MAX).astype(np.int64)
    return np.repeat(np.repeat(e, high, axis=0), BLOCK, axis=1)[:rows, :cols]


def quantise(x, square=False):
    """The values that x [rows][cols] stands for in 8 bits, groups along its rows."""
    x = np.asarray(x, np.float64)
    grid = e4m3_numbers()
    unit = np.ldexp(1.0, exponents(x, square))
    a = np.where(np.isfinite(x), np.abs(x), 0.0) / unit
    hi = np.clip(np.searchsorted(grid, a), 1, grid.size - 1)
    below, above = a - grid[hi - 1], grid[hi] - a
    code = np.where((below < above) | ((below == above) & ((hi - 1) % 2 == 0)), hi - 1, hi)
    return np.where(np.isfinite(x), np.copysign(grid[code], x) * unit, np.nan)


def gelu(z):
    return 0.5 * z * (1.0 + np.tanh(np.sqrt(2.0 / np.pi) * (z + 0.044715 * z ** 3)))


def matmul(a, b, bias=None):
    """(C, the sum of its products' magnitudes) for values a [M][K], b [N][K]."""
    c = np.asarray(a, np.float64) @ np.asarray(b, np.float64).T
    size = np.abs(a) @ np.abs(b).T
    return (c if bias is None else c + np.asarray(bias, np.float64)), size
