"""The 8-bit operators from their definitions, in 64 bits on the host (numpy).

Codes are uint8 arrays holding OCP E4M3 numbers; the format's values come from
its bit fields here, not from any library's conversion.  Shares no code with the
HIP path.
"""
import numpy as np

GROUP = 128
LARGEST = 448.0
SMALLEST_SCALE = 2.0 ** -126


def _values():
    v = np.empty(256)
    for c in range(256):
        sign, exponent, mantissa = c >> 7, (c >> 3) & 15, c & 7
        if exponent == 15 and mantissa == 7:
            x = np.nan
        elif exponent == 0:
            x = mantissa * 2.0 ** -9
        else:
            x = (8 + mantissa) * 2.0 ** (exponent - 10)
        v[c] = -x if sign else x
    return v


VALUES = _values()
_POSITIVE = VALUES[:127]  # 0 to 448, ascending


def round_to_code(q):
    """Codes of the nearest numbers, ties to the even code, at most the largest; NaN and infinities to NaN."""
    q = np.asarray(q, dtype=np.float64)
    a = np.where(np.isfinite(q), np.minimum(np.abs(q), LARGEST), 0.0)
    above = np.minimum(np.searchsorted(_POSITIVE, a), 126)
    below = np.maximum(above - 1, 0)
    up, down = _POSITIVE[above] - a, a - _POSITIVE[below]
    code = np.where(up < down, above, np.where(up > down, below, np.where(above % 2 == 0, above, below)))
    code = np.where(np.isfinite(q), code, 127)
    return (code | np.where(np.signbit(q), 128, 0)).astype(np.uint8)


def group_scales(y, tile_rows):
    """32-bit scales of the groups of y (64 bits), [row groups, column groups]."""
    rows, cols = y.shape
    out = np.empty((-(-rows // tile_rows), -(-cols // GROUP)), dtype=np.float32)
    for i in range(out.shape[0]):
        for j in range(out.shape[1]):
            a = np.abs(y[i * tile_rows:(i + 1) * tile_rows, j * GROUP:(j + 1) * GROUP])
            top = a[np.isfinite(a)].max(initial=0.0)
            out[i, j] = max(top / LARGEST, SMALLEST_SCALE) if top > 0 else 1.0
    return out


def spread(scales, tile_rows, rows, cols):
    """A scale for every element, in 64 bits."""
    s = np.repeat(np.asarray(scales, dtype=np.float64), tile_rows, 0)[:rows]
    return np.repeat(s, GROUP, 1)[:, :cols]


def rms_norm(x, residual, weight, eps):
    """(y, h): h = x + residual rounded to 32 bits, as the operator forms it."""
    h = np.asarray(x, dtype=np.float32)
    if residual is not None:
        h = h + np.asarray(residual, dtype=np.float32)
    h64 = h.astype(np.float64)
    return h64 / np.sqrt((h64 * h64).mean(1, keepdims=True) + eps) * np.asarray(weight, dtype=np.float64), h


def gated(gate, up):
    g = np.asarray(gate, dtype=np.float64)
    with np.errstate(over="ignore"):
        return g / (1 + np.exp(-g)) * np.asarray(up, dtype=np.float64)


def matmul(a, a_scales, b, b_scales):
    """(c, size): the product, and the sum of its terms' magnitudes, which bounds how far rounding can move it."""
    x = VALUES[a] * spread(a_scales, 1, *a.shape)
    y = VALUES[b] * spread(b_scales, GROUP, *b.shape)
    return x @ y.T, np.abs(x) @ np.abs(y).T


def adapters(y, x, x_scales, down, up, index, factors):
    """(out, size): y with each token's adapter in 64 bits, and the sum of its terms' magnitudes."""
    out, size = np.array(y, dtype=np.float64), np.abs(np.asarray(y, dtype=np.float64))
    numbers = VALUES[x] * spread(x_scales, 1, *x.shape)
    for t, a in enumerate(index):
        if 0 <= a < len(down):
            inner = down[a] @ numbers[t]
            out[t] += factors[a] * (up[a] @ inner)
            size[t] += abs(factors[a]) * (np.abs(up[a]) @ (np.abs(down[a]) @ np.abs(numbers[t])))
    return out, size
