"""The products' bounds let nothing go missing: mistakes planted in the oracle are refused, on the CPU."""
import numpy as np
import pytest
import torch

import fp8_bounds as bounds
from oracle import fp8
from paper_2510_23938_amd import hv  # noqa: E402  (a missing library fails the run, never skips it)

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ZERO = 0  # the code of 0


def rounded(c, dtype):
    return torch.from_numpy(c).to(TYPES[dtype]).double().numpy()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", bounds.LONG)
def test_a_right_product_passes_and_a_wrong_one_does_not(m, n, k, dtype):
    near = dtype != "f32"
    a, sa, b, sb = bounds.operands(m, n, k, near)
    c, spread = bounds.exact(a, sa, b, sb)
    bounds.check(rounded(c, dtype), c, spread, k, dtype, near)

    def refused(a=a, sa=sa, b=b, sb=sb):
        with pytest.raises(AssertionError):
            bounds.check(rounded(bounds.exact(a, sa, b, sb)[0], dtype), c, spread, k, dtype, near)

    def without(first, last):
        lost = a.copy()
        lost[:, first:last] = ZERO
        return lost

    groups = -(-k // 128)
    refused(a=without(k - 1, k))                    # the last column
    refused(a=without(0, 1))                        # the first
    refused(a=without((groups - 1) * 128, k))       # the last group, whole or not
    for aligned in (True, False):                   # one of the parts that the columns are split into
        parts = hv.matmul_launches(m, n, k, TYPES[dtype], aligned)[-1][3]
        if parts > 1:
            each = -(-groups // parts) * 128
            refused(a=without(each, 2 * each))
            refused(a=without((parts - 1) * each, k))
    if groups > 1:
        late = sa.copy()
        late[:, 1:] = sa[:, :-1]                    # the group before's scales
        refused(sa=late)
    one = b.copy()
    one[n // 2, k // 2] ^= 0x80                     # one code's sign, in one column of the result
    refused(b=one)


@pytest.mark.parametrize("m,n,k", bounds.LONG)
def test_a_32_bit_result_of_16_bit_sums_does_not_pass(m, n, k):
    """What the matrix unit drops of 16 products, 1.5e-5 of a typical sum, is seen in a 32-bit result."""
    a, sa, b, sb = bounds.operands(m, n, k, False)
    c, spread = bounds.exact(a, sa, b, sb)
    noise = np.random.default_rng(1).standard_normal(c.shape) * 1.5e-5 * spread
    with pytest.raises(AssertionError):
        bounds.check(rounded(c + noise, "f32"), c, spread, k, "f32", False)


def test_spread_is_the_root_of_the_terms_squares():
    a, sa, b, sb = bounds.operands(3, 5, 300, False)
    c, spread = bounds.exact(a, sa, b, sb)
    terms = np.array([fp8.VALUES[a[1, t]] * sa[1, t // 128] * fp8.VALUES[b[4, t]] * sb[0, t // 128]
                      for t in range(300)])
    assert np.isclose(c[1, 4], terms.sum()) and np.isclose(spread[1, 4], np.sqrt((terms ** 2).sum()))
