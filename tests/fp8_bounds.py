"""What a product of 8-bit matrices may differ by from its value in 64 bits, by the additions that an output goes
through and not by its columns, so that a lost column, group or part of the columns cannot hide in it.

* An output's terms pass at most 128 additions within a group (the 32-bit path's four instructions of 32 columns),
  one for each group, and 72 where waves' or parts' sums meet.  Each is off by at most 2^-24 of a partial sum, the
  scales' products and the results' scaling by a few 2^-24 more.  The operands here have no preferred sign, so
  partial sums are about as large as the root of the terms' squares, ``spread``, and the errors are independent: a
  standard deviation of (sqrt(additions) + 4) * 2^-24 * spread at most, six of them for a single output.
* 16-bit results: what the matrix unit drops of 16 products is below 2^-13 of the largest of them each.  Of codes of
  four binades (``near``) that is nothing, of ordinary ones 2^-14 of the spread as a whole, six times that for one
  output.
* The result's own rounding: half an ulp for one output, and for all of them together no more than a uniformly
  distributed one's standard deviation, half an ulp divided by sqrt(3).
"""
import numpy as np

from oracle import fp8

HALF_ULP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}

# few rows, columns in parts, odd addresses, remainders of every kind
LONG = [(1, 1000, 20479), (4, 515, 9001), (8, 130, 28672), (16, 130, 20003), (17, 2000, 4100), (24, 500, 8192),
        (40, 300, 9000), (96, 1024, 8192), (100, 130, 20000), (130, 130, 11008), (333, 500, 2777), (300, 1100, 1280)]


def operands(m, n, k, near, seed=31):
    """(a, a_scales, b, b_scales): codes without a preferred sign, scales that let every group count."""
    rng = np.random.default_rng([m, n, k, seed])

    def codes(rows):
        if near:
            return (rng.integers(12 << 3, 127, (rows, k)) | rng.integers(0, 2, (rows, k)) << 7).astype(np.uint8)
        return fp8.round_to_code(np.clip(rng.standard_normal((rows, k)) * 60, -448, 448))

    g = -(-k // 128)
    return (codes(m), np.exp2(rng.uniform(-10, -9, (m, g))).astype(np.float32), codes(n),
            np.exp2(rng.uniform(-10, -9, (-(-n // 128), g))).astype(np.float32))


def exact(a, a_scales, b, b_scales):
    """(c, spread) in 64 bits."""
    x = fp8.VALUES[a] * fp8.spread(a_scales, 1, *a.shape)
    y = fp8.VALUES[b] * fp8.spread(b_scales, 128, *b.shape)
    return x @ y.T, np.sqrt((x * x) @ (y * y).T)


def check(got, c, spread, k, dtype, near):
    assert got.shape == c.shape and np.isfinite(got).all()
    sums = (np.sqrt(128 + -(-k // 128) + 72) + 4) * 2.0 ** -24 + (0 if near or dtype == "f32" else 2.0 ** -14)
    smallest = 2.0 ** -25 if dtype == "f16" else 0  # half of half precision's smallest number
    off = np.abs(got - c)
    one = off - (6 * sums * spread + HALF_ULP[dtype] * np.abs(c) + smallest)
    assert (one <= 0).all(), (np.argwhere(one > 0)[:5], one.max())
    if c.size >= 500:
        whole = np.hypot(HALF_ULP[dtype] / np.sqrt(3) * np.linalg.norm(c) + smallest * np.sqrt(c.size),
                         sums * np.linalg.norm(spread))
        assert np.linalg.norm(off) <= whole, (np.linalg.norm(off), whole)
