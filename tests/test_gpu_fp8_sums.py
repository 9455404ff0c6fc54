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
