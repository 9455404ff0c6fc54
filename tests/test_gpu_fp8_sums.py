"""The product's sums (hv_fp8_matmul), within bounds that no lost column, group or part could pass (fp8_bounds.py;
test_fp8_bounds.py plants such mistakes in the oracle)."""
import numpy as np
import pytest
import torch

import fp8_bounds as bounds
import test_gpu_fp8 as base
from paper_2510_23938_amd import hv  # noqa: E402  (a missing library fails the run, never skips it)

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
TYPES = base.TYPES


def on_gpu(a, sa, b, sb, pad=0, offset=0):
    return (base.codes_on_gpu(a, pad, offset), torch.from_numpy(sa).to(DEV), base.codes_on_gpu(b, pad, offset),
            torch.from_numpy(sb).to(DEV))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", bounds.LONG)
def test_long_sums_lose_nothing(m, n, k, dtype):
    near = dtype != "f32"
    host = bounds.operands(m, n, k, near)
    c, spread = bounds.exact(*host)
    for pad, offset in ((-k % 16, 0), (0, 0), (3, 5)):  # aligned rows; as they are; odd addresses
        got = hv.hv_fp8_matmul(*on_gpu(*host, pad, offset), TYPES[dtype]).double().cpu().numpy()
        bounds.check(got, c, spread, k, dtype, near)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(9, 4000, 1100), (250, 260, 1023), (520, 2050, 900), (2300, 8200, 260)])
def test_sums_of_ordinary_codes(m, n, k, dtype):
    host = bounds.operands(m, n, k, False)
    c, spread = bounds.exact(*host)
    got = hv.hv_fp8_matmul(*on_gpu(*host), TYPES[dtype]).double().cpu().numpy()
    bounds.check(got, c, spread, k, dtype, False)


def dropped(a, sa, b, sb):
    """The most that the matrix unit may drop for a 16-bit result: of each 16 neighbouring columns' products 15 that
    are off by up to 2^-13 of the largest."""
    x = np.abs(bounds.fp8.VALUES[a]) * bounds.fp8.spread(sa, 1, *a.shape)
    y = np.abs(bounds.fp8.VALUES[b]) * bounds.fp8.spread(sb, 128, *b.shape)
    total = np.zeros((len(a), len(b)))
    for t in range(0, a.shape[1], 16):
        total += (x[:, None, t:t + 16] * y[None, :, t:t + 16]).max(2)
    return 15 * 2.0 ** -13 * total


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("strong", ["far above", "cancelling"])
@pytest.mark.parametrize("m,n,k", [(3, 200, 1100), (40, 300, 500), (150, 256, 777)])
def test_a_few_strong_columns(m, n, k, strong, dtype):
    """Columns of 448 among small codes, or pairs of them that cancel, in every 16 columns: 16-bit results lose what
    the header says and no more, 32-bit results nothing."""
    rng = np.random.default_rng([m, n, k, 41])
    a, sa, b, sb = bounds.operands(m, n, k, False)
    a = (a & 0x80) | (a & 0x7f) // 2  # magnitudes below 2
    first = np.arange(0, k - 15, 16)
    at = first + rng.integers(0, 8, len(first))
    a[:, at], b[:, at] = 126, 126
    if strong == "cancelling":
        a[:, at + 5], b[:, at + 5] = 126 | 128, 126
    c, spread = bounds.exact(a, sa, b, sb)
    got = hv.hv_fp8_matmul(*on_gpu(a, sa, b, sb), TYPES[dtype]).double().cpu().numpy()
    # sums pass terms as large as the strong columns' whole sum, so that its size stands for the partial sums'
    size = np.abs(bounds.fp8.VALUES[a] * bounds.fp8.spread(sa, 1, *a.shape)) @ \
        np.abs(bounds.fp8.VALUES[b] * bounds.fp8.spread(sb, 128, *b.shape)).T
    allowed = (128 + -(-k // 128) + 72) * 2.0 ** -24 * size + bounds.HALF_ULP[dtype] * np.abs(c)
    allowed += 0 if dtype == "f32" else dropped(a, sa, b, sb) + (2.0 ** -25 if dtype == "f16" else 0)
    off = np.abs(got - c) - allowed
    assert (off <= 0).all(), (np.argwhere(off > 0)[:5], off.max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n,k", [(5, 300, 200), (30, 200, 300), (300, 300, 256)])
def test_scales_whose_product_is_the_smallest_normal_number(m, n, k, dtype):
    """Down to 2^-126 nothing is lost: the result times a power of two, bit for bit.  Two scales of 2^-75 have a
    product of zero."""
    a, _, b, _ = bounds.operands(m, n, k, True)  # products are multiples of 16, sums below 2^24 of them
    ones_a, ones_b = (np.ones((-(-r // h), -(-k // 128)), np.float32) for r, h in ((m, 1), (n, 128)))
    want = hv.hv_fp8_matmul(*on_gpu(a, ones_a, b, ones_b), TYPES[dtype])
    assert want.abs().max() > 0
    for p, q in ((-70, -56), (-126, 0), (0, -126), (-1, -125)):
        got = hv.hv_fp8_matmul(*on_gpu(a, ones_a * np.float32(2.0 ** p), b, ones_b * np.float32(2.0 ** q)), TYPES[dtype])
        assert torch.equal(got.double() * 2.0 ** 126, want.double())
    tiny_a, tiny_b = ones_a * np.float32(2.0 ** -75), ones_b * np.float32(2.0 ** -75)
    assert (hv.hv_fp8_matmul(*on_gpu(a, tiny_a, b, tiny_b), TYPES[dtype]) == 0).all()
