"""Oracle of the 8-bit key/value cache (float64 NumPy): what a cache holds after a
write, and attention over it.

Tokens of a segment are grouped in blocks of 64 from its first one.  A block of
one head keeps its keys, and likewise its values, as e4m3 numbers (4 significant
bits, smallest step 2^-9, largest 448) times 2^e: with A their largest finite
magnitude, e is the smallest integer with A <= 448 2^e, held in -100 .. 119.
"""
import numpy as np

BLOCK = 64
E_MIN, E_MAX = -100, 119


def e4m3_numbers() -> np.ndarray:
    """The non-negative finite e4m3 numbers, ascending (index = code)."""
    sub = [m / 512.0 for m in range(8)]
    normal = [(1.0 + m / 8.0) * 2.0 ** x for x in range(-6, 9) for m in range(8)]
    return np.array((sub + normal)[:127])  # the 128th code is NaN


def round_e4m3(y: np.ndarray) -> np.ndarray:
    """Nearest e4m3 number, ties to the even code; past 448 saturated, NaN where y is not finite."""
    grid = e4m3_numbers()
    y = np.asarray(y, np.float64)
    a = np.where(np.isfinite(y), np.abs(y), 0.0)
    hi = np.clip(np.searchsorted(grid, a), 1, grid.size - 1)
    lo = hi - 1
    below, above = a - grid[lo], grid[hi] - a
    code = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    return np.where(np.isfinite(y), np.copysign(grid[code], y), np.nan)


def block_exponent(x: np.ndarray) -> int:
    f = np.abs(x[np.isfinite(x)])
    top = float(f.max()) if f.size else 0.0
    e = E_MIN
    while top > 448.0 * 2.0 ** e and e < E_MAX:
        e += 1
    return e


def blocks(bounds):
    """(first token, end) of every block of segments with the given token bounds."""
    out = []
    for a, b in zip(bounds[:-1], bounds[1:]):
        out += [(t, min(int(b), t + BLOCK)) for t in range(int(a), int(b), BLOCK)]
    return out


def quantise(x: np.ndarray, bounds) -> np.ndarray:
    """The values that a cache with contents x [N][heads][d] holds."""
    x = np.asarray(x, np.float64)
    out = np.empty_like(x)
    for a, b in blocks(bounds):
        for h in range(x.shape[1]):
            e = block_exponent(x[a:b, h])
            out[a:b, h] = round_e4m3(x[a:b, h] / 2.0 ** e) * 2.0 ** e
    return out


def write(held: np.ndarray, rows: np.ndarray, idx: np.ndarray, bounds) -> np.ndarray:
    """The values held after rows [n][heads][d] are written at tokens idx: blocks that no row falls into are left
    alone (a token outside the cache is skipped, the last of several rows for a token counts)."""
    x = np.array(held, np.float64)
    touched = np.zeros(x.shape[0], bool)
    for j, t in enumerate(idx):
        if 0 <= t < x.shape[0]:
            x[t] = rows[j]
            touched[t] = True
    q = quantise(x, bounds)
    for a, b in blocks(bounds):
        if not touched[a:b].any():
            q[a:b] = held[a:b]
    return q


def attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, cu_q, cu_kv, kv_len=None):
    """Base-2 softmax attention, q [n][heads][d], k and v [N][kv_heads][d]; zeros where there are no keys.  Also returns
    sum_t w |v| (w the softmax weights) and the largest sum over dims of |q k|, which bound rounding errors."""
    n, heads, d = q.shape
    group = heads // k.shape[1]
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    big = np.zeros((n, heads, 1))
    for i in range(len(cu_q) - 1):
        a, b, k0 = int(cu_q[i]), int(cu_q[i + 1]), int(cu_kv[i])
        k1 = int(cu_kv[i + 1]) if kv_len is None else k0 + int(kv_len[i])
        if a == b or k0 == k1:
            continue
        for h in range(heads):
            kh, vh = k[k0:k1, h // group], v[k0:k1, h // group]
            s = q[a:b, h] @ kh.T
            w = np.exp2(s - s.max(axis=1, keepdims=True))
            w /= w.sum(axis=1, keepdims=True)
            out[a:b, h] = w @ vh
            mag[a:b, h] = w @ np.abs(vh)
            big[a:b, h, 0] = (np.abs(q[a:b, h]) @ np.abs(kh).T).max(axis=1)
    return out, mag, big
