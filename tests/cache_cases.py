"""Batches and caches for the tests of the 8-bit cache: a host copy for the oracle beside the GPU's."""
import numpy as np
import torch

from oracle import fp8, fp8_cache
from paper_2510_23938_amd import hv  # noqa: E402  (a missing library fails the run, never skips it)

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


class Batch:
    """Sequences of (new tokens, tokens in all), their pages drawn without order from a pool with some to spare."""

    def __init__(self, rng, sequences, page, spare=3, columns=0, device="cuda"):
        new, self.lengths = (np.array(a, dtype=np.int32) for a in zip(*sequences)) if sequences else \
            (np.zeros(0, np.int32),) * 2
        self.starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        counts = -(-self.lengths // page)
        self.pool = int(counts.sum()) + spare
        order = rng.permutation(self.pool).astype(np.int32)
        self.table = np.full((len(new), max(int(counts.max(initial=0)), columns, 1)), -1, dtype=np.int32)
        at = 0
        for i, n in enumerate(counts):
            self.table[i, :n] = order[at:at + n]
            at += n
        self.tokens = int(self.starts[-1])
        self.device = device

    def gpu(self):
        return tuple(torch.from_numpy(a).to(self.device) for a in (self.starts, self.lengths, self.table))


def random_cache(rng, pages, heads, page, dim, spread=3.0):
    """An oracle cache of random codes and scales of several binades."""
    blocks = page // 16

    def codes(shape):
        return fp8.round_to_code(np.clip(rng.standard_normal(shape) * 100, -448, 448))

    def scales():
        return np.exp2(np.round(rng.uniform(-spread, spread, (pages, heads, blocks)) - 7)).astype(np.float32)

    return fp8_cache.Cache(codes((pages, heads, page, dim)), scales(), codes((pages, heads, blocks, dim, 16)), scales())


def on_gpu(cache, k_pad=0, v_pad=0, device="cuda"):
    """The same cache as hv.Fp8Cache; pads are bytes between heads, and twice as many between pages.  What lies between
    is NaN."""
    def codes(a, pad):
        pages, heads = a.shape[:2]
        inner = int(np.prod(a.shape[2:]))
        head = inner + pad
        page = heads * head + pad
        raw = torch.full((pages * page + 16,), 0x7f, dtype=torch.uint8, device=device)
        strides = (page, head, a.shape[3], 1) if a.ndim == 4 else (page, head, a.shape[3] * 16, 16, 1)
        t = raw.as_strided(a.shape, strides)
        t.copy_(torch.from_numpy(a).to(device))
        return t.view(torch.float8_e4m3fn)

    return hv.Fp8Cache(codes(cache.k, k_pad), torch.from_numpy(cache.ks).to(device), codes(cache.v, v_pad),
                       torch.from_numpy(cache.vs).to(device))


def host_tensors(cache):
    """(k, ks, v, vs) of an hv.Fp8Cache as numpy arrays, codes as bytes."""
    return tuple(t.view(torch.uint8).cpu().numpy() if t.dtype == torch.float8_e4m3fn else t.cpu().numpy()
                 for t in cache.tensors())
