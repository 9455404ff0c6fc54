"""What attention over the 8-bit cache may differ by from its value in 64 bits.

* Scores.  The products of 16-bit queries and codes are exact in 32 bits; a sum of up to 256 of them, its product with
  the scales and the subtraction of the row's maximum pass at most 256 + 3 roundings of 2^-24 of a partial sum, which
  ``steep`` (the largest sum of magnitudes) bounds, each of its own sign: 6 standard deviations of the root of their
  number are below 2^-24 * 100.  A weight is off relatively by that error (the maximum's part is common to all), and by
  the exponential's, below 2^-21.
* Weights are added in 32 bits in order, at most 2^-24 for each of up to 2^12 additions in a lane's own sum (below
  2^-18 as a whole in the tests, whose errors are independent), and multiplied with values in 32 bits.
* A weight is rounded to the type: half a step each, uniform and independent, so an output is off by half a step
  / sqrt(3) of ``root`` (the root of the sum of (w v)^2) as a standard deviation; six of them.  For half precision weights
  below 2^-14 of the largest lose up to 2^-25 of it each.
* The result is rounded once.
"""
import numpy as np

HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}


def check(got, want, dtype, keys):
    """``want``: what oracle.attention gives; ``keys``: the most that a row sees."""
    out, size, root, steep = want
    rows = ~np.isnan(out).all((1, 2))
    got, out, size, root, steep = got[rows], out[rows], size[rows], root[rows], steep[rows]
    bad = np.isnan(out)
    assert np.array_equal(np.isnan(got), bad)
    weights = 2 * (100 * 2.0 ** -24 * steep + 2.0 ** -21 + 2.0 ** -18)[:, :, None]
    half = HALF_STEP[dtype]
    allowed = weights * size + 6 * half / np.sqrt(3) * root + half * np.abs(out)
    if dtype == "f16":
        largest = np.nanmax(size, initial=0.0)
        allowed += 2.0 ** -25 * (1 + keys * largest * 4)
    off = np.abs(got - out)
    worse = ~(off <= allowed) & ~bad
    assert not worse.any(), (np.argwhere(worse)[:5], np.nanmax(off - allowed), np.nanmax(off / np.maximum(allowed, 1e-300)))
