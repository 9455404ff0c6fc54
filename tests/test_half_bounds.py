"""The bounds of half precision let nothing go missing among 20,000 keys: mistakes planted in the oracle, on the CPU."""
import numpy as np
import pytest
import torch

import half_bounds
from cache_cases import Batch, random_cache
from oracle import fp8_cache


@pytest.mark.parametrize("sequences", [[(1, 20000)], [(3, 900)]], ids=str)
@pytest.mark.parametrize("spread", [0.0, 3.0])
def test_lost_blocks_are_seen(sequences, spread):
    rng = np.random.default_rng([sequences[0][1], int(spread)])
    batch = Batch(rng, sequences, 64, device="cpu")
    cache = random_cache(rng, batch.pool, 2, 64, 64, spread)
    q = torch.from_numpy(rng.standard_normal((batch.tokens, 4, 64)) * 0.1).to(torch.float16).double().numpy()
    at = batch.starts, batch.lengths, batch.table, 0.125
    want, lost = fp8_cache.attention(cache, q, *at), half_bounds.subnormal_losses(cache, q, *at)

    def rounded(x):
        return torch.from_numpy(x).half().double().numpy()

    half_bounds.check(rounded(want[0]), want, lost)
    largest = max(range(0, int(batch.lengths[0]) // 16), key=lambda b: cache.vs[batch.table[0, b // 4], 0, b % 4])
    page, block = batch.table[0, largest // 4], largest % 4
    for change in ("values", "scale", "keys"):
        wrong = cache.copy()
        if change == "values":
            wrong.v[page, 0, block] = 0
        elif change == "scale":
            wrong.vs[page, 0, block] *= 2
        else:
            wrong.k[page, 0, block * 16:block * 16 + 16] ^= 0x80
            wrong.ks[page, 0, block] *= 64
        with pytest.raises(AssertionError):
            half_bounds.check(rounded(fp8_cache.attention(wrong, q, *at)[0]), want, lost)
