"""Attention in half precision against its definition in 64 bits, within bounds of each row (half_bounds.py)."""
import numpy as np
import pytest
import torch

import half_bounds
from cache_cases import Batch, on_gpu, random_cache
from oracle import fp8_cache
from paper_2510_23938_amd import hv  # noqa: E402  (a missing library fails the run, never skips it)

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")


@pytest.mark.parametrize("steep", [0.1, 1.0, 8.0])
@pytest.mark.parametrize("spread", [0.0, 3.0, 6.0])
@pytest.mark.parametrize("sequences", [[(1, 20000), (1, 300)], [(6, 5000), (6, 70)], [(40, 2000), (40, 40)]], ids=str)
def test_half_precision(sequences, spread, steep):
    rng = np.random.default_rng([len(sequences), sequences[0][0], int(spread), int(10 * steep)])
    batch = Batch(rng, sequences, 64)
    host = random_cache(rng, batch.pool, 2, 64, 64, spread)
    q = torch.from_numpy(rng.standard_normal((batch.tokens, 8, 64)) * steep).to(torch.float16)
    out = hv.hv_fp8_attention(q.to(DEV), on_gpu(host), *batch.gpu()).double().cpu().numpy()
    args = host, q.double().numpy(), batch.starts, batch.lengths, batch.table, 0.125
    half_bounds.check(out, fp8_cache.attention(*args), half_bounds.subnormal_losses(*args))
