"""The 8-bit operators at the ends of their ranges, against their definitions in 64 bits (oracle/fp8.py), and
their calls on other streams, with shared scratch and with rows far apart."""
import numpy as np
import pytest
import torch

import test_gpu_fp8 as base
from oracle import fp8
from paper_2510_23938_amd import hv  # noqa: E402  (a missing library fails the run, never skips it)

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
TYPES = base.TYPES


@pytest.mark.parametrize("dtype", TYPES)
def test_gated_by_a_closing_gate(dtype):
    """exp(-gate) leaves 32 bits at -88.7, and its reciprocal is subnormal from -87.3 on, while the gate's product
    with a large factor is an ordinary number.  Two exponentials of half the gate, each within an ulp, and three
    products stay below the bound on y's relative error."""
    up = 6e4 if dtype == "f16" else 1e36
    last = -96 if dtype == "f16" else -150  # y stays above the smallest scale's 448
    gate = np.linspace(-80, last, 12)[:, None] + np.linspace(0, 3, 300)[None, :]  # groups of neighbouring gates
    mixed = np.linspace(last, 4, 300)[None, :] * np.ones((4, 1))                  # and of all
    rng = np.random.default_rng(21)
    g = base.on_gpu(np.concatenate([gate, mixed]), TYPES[dtype])
    u = base.on_gpu(up * rng.uniform(0.25, 1, (16, 300)) * rng.choice([-1, 1], (16, 300)), TYPES[dtype])
    codes, scales = hv.hv_fp8_gated(g, u)
    y = fp8.gated(g.double().cpu().numpy(), u.double().cpu().numpy())
    got = scales.cpu().numpy()
    want = fp8.group_scales(y, 1)
    assert (want > 2.0 ** -126).all()
    assert np.all(np.abs(got / want - 1) <= base.Y_ERROR)
    base.check_codes(base.bytes_of(codes), y, got, 1, 2 * base.Y_ERROR)
