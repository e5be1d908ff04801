"""8-bit rows in float64 on the CPU, from the format's definition (see include/moeca_q8.h).

A row is held as values on the 8-bit format's grid and one power-of-two scale
per 128 of them.  Nothing here goes through a float8 type: the grid is
worked out from the formats' significand and exponent widths.
"""
import numpy as np

BLOCK = 128
# name: (largest value, significand digits after the point, least normal exponent, has infinities)
FORMATS = {"e4m3": (448.0, 3, -6, False), "e5m2": (57344.0, 2, -14, True)}


def blocks(width: int) -> int:
    return -(-width // BLOCK)


def to_grid(y, fmt: str):
    """Nearest value of the format, ties to even; |y| at most the largest, or not finite."""
    most, digits, least, inf = FORMATS[fmt]
    y = np.asarray(y, np.float64)
    fin = np.where(np.isfinite(y), y, 0.0)
    exp = np.maximum(np.frexp(fin)[1] - 1, least)  # |y| in [2^exp, 2^(exp + 1)), or below the normals
    step = np.ldexp(1.0, exp - digits)
    out = np.rint(fin / step) * step
    out = np.where(np.isnan(y), np.nan, out)
    return np.where(np.isinf(y), y if inf else np.nan, out)


def quantise(x, fmt: str):
    """Rows of x [n, width]: (grid values [n, width], scale exponents [n, blocks])."""
    most = FORMATS[fmt][0]
    x = np.asarray(x, np.float64)
    n, width = x.shape
    q, e = np.empty_like(x), np.zeros((n, blocks(width)), np.int64)
    for b in range(blocks(width)):
        part = x[:, b * BLOCK:(b + 1) * BLOCK]
        a = np.where(np.isfinite(part), np.abs(part), 0.0).max(1)
        m, ex = np.frexp(a / most)  # a / most = m 2^ex, m in [1/2, 1): most is 7 x 2^j, so the division may round
        ex = np.where(m == 0.5, ex - 1, ex)
        ex = np.where(a > most * np.ldexp(1.0, ex), ex + 1, ex)
        ex = np.where((a > 0) & (a <= most * np.ldexp(1.0, ex - 1)), ex - 1, ex)
        e[:, b] = np.where(a > 0, np.maximum(ex, -127), 0)
        q[:, b * BLOCK:(b + 1) * BLOCK] = to_grid(part * np.ldexp(1.0, -e[:, b])[:, None], fmt)
    return q, e


def dequantise(q, e):
    width = q.shape[-1]
    return np.asarray(q, np.float64) * np.ldexp(1.0, np.asarray(e))[..., np.arange(width) // BLOCK]


def combine(h, rows, weights, x=None, gate=None, seq=1):
    """Eq. 8 over rows h [R, D]; an entry of rows outside [0, R) holds nothing.  Returns (out, norms)."""
    T, k = rows.shape
    live = (rows >= 0) & (rows < len(h))
    hv = np.where(live[..., None], h[np.where(live, rows, 0)], 0.0)
    w = np.where(live, 1.0 if weights is None else weights, 0.0)
    y = (w[..., None] * hv).sum(1)
    if gate is not None:
        y = np.asarray(gate, np.float64)[np.arange(T) // seq] * y
    if x is not None:
        y = np.asarray(x, np.float64) + y
    return y, np.sqrt((hv * hv).sum(-1))


def gelu(z, tanh_form: bool):
    from scipy.special import erf
    z = np.asarray(z, np.float64)
    if tanh_form:
        return 0.5 * z * (1 + np.tanh(np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3)))
    return 0.5 * z * (1 + erf(z / np.sqrt(2)))


def matmul(a, b, offsets, n_cols, bias=None, act="none"):
    """Grouped product of dequantised rows a [M, K] and b [G n_cols, K]: (result [M, n_cols], rows computed [M],
    sum_k |a b| + |bias| [M, n_cols], the scale of the fp32 sum's error)."""
    M = len(a)
    out, big = np.zeros((M, n_cols)), np.zeros((M, n_cols))
    done = np.zeros(M, bool)
    off = np.clip(np.asarray(offsets), 0, M)
    for g in range(len(off) - 1):
        lo, hi = off[g], off[g + 1]
        if hi <= lo:
            continue
        w = b[g * n_cols:(g + 1) * n_cols]
        z = a[lo:hi] @ w.T
        big[lo:hi] = np.abs(a[lo:hi]) @ np.abs(w).T
        if bias is not None:
            z = z + bias[g]
            big[lo:hi] += np.abs(bias[g])
        out[lo:hi] = z if act == "none" else gelu(z, act == "gelu_tanh")
        done[lo:hi] = True
    return out, done, big
