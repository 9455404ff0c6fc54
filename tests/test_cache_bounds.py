"""The bounds of the attention and the adapters let nothing go missing: mistakes planted in the oracle are refused, on
the CPU.  And the cache's oracle against what it is not made from."""
import numpy as np
import pytest
import torch

import cache_bounds
import test_gpu_fp8_adapters as adapters_test
from cache_cases import Batch, random_cache
from oracle import fp8, fp8_cache

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def rounded(x, dtype):
    return torch.from_numpy(x).to(TYPES[dtype]).double().numpy()


def case(sequences, heads=4, kv_heads=2, dim=64, page=32, dtype="bf16", seed=1):
    rng = np.random.default_rng(seed)
    batch = Batch(rng, sequences, page, device="cpu")
    cache = random_cache(rng, batch.pool, kv_heads, page, dim, 1.0)
    q = torch.from_numpy(rng.standard_normal((batch.tokens, heads, dim)) * 0.1).to(TYPES[dtype]).double().numpy()
    return batch, cache, q


def attention(batch, cache, q, lengths=None, table=None, scale=0.125, window=0, sinks=0):
    return fp8_cache.attention(cache, q, batch.starts, batch.lengths if lengths is None else lengths,
                               batch.table if table is None else table, scale, window, sinks)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sequences", [[(1, 600), (1, 130)], [(9, 900)], [(40, 300), (1, 40)]], ids=str)
def test_a_right_attention_passes_and_a_wrong_one_does_not(sequences, dtype):
    batch, cache, q = case(sequences, dtype=dtype)
    window, sinks = 100, 4
    whole = attention(batch, cache, q)
    seen = attention(batch, cache, q, window=window, sinks=sinks)
    keys = int(batch.lengths.max())
    cache_bounds.check(rounded(whole[0], dtype), whole, dtype, keys)
    cache_bounds.check(rounded(seen[0], dtype), seen, dtype, keys)

    def refused(want, wrong):
        with pytest.raises(AssertionError):
            cache_bounds.check(rounded(wrong[0], dtype), want, dtype, keys)

    refused(whole, attention(batch, cache, q, lengths=batch.lengths - 1))               # all a token off
    refused(seen, attention(batch, cache, q, window=window + 1, sinks=sinks))           # a window one longer
    refused(seen, attention(batch, cache, q, window=window - 1, sinks=sinks))
    refused(seen, attention(batch, cache, q, window=window, sinks=sinks + 1))           # a first token more
    refused(seen, attention(batch, cache, q, window=window, sinks=0))
    refused(whole, attention(batch, cache, q, scale=0.125 * 1.3))
    swapped = batch.table.copy()
    swapped[:, [0, 1]] = swapped[:, [1, 0]]
    refused(seen, attention(batch, cache, q, table=swapped, window=window, sinks=sinks))  # other pages among the first
    refused(whole, attention(batch, cache, q[:, ::-1].copy()))                          # heads the other way
    for part in ("k", "v", "ks", "vs"):                                                 # a page's codes, scales
        wrong = cache.copy()
        page = batch.table[0, 2]
        if part == "k":
            wrong.k[page, 0] ^= 0x80
        elif part == "v":
            wrong.v[page, 0, 0, 3] = 0x7e
        elif part == "ks":
            wrong.ks[page, 0] *= 4
        else:
            wrong.vs[page, 0, 0] *= 2
        refused(whole, attention(batch, wrong, q))
    lost = cache.copy()                                                                 # a tile of 64 keys lost
    for position in range(64, 128):
        lost.k[batch.table[0, position // 32], :, position % 32] = 0
    refused(whole, attention(batch, lost, q))


@pytest.mark.parametrize("sequences,window,sinks", [([(3, 50), (1, 1), (7, 7)], 0, 0), ([(5, 90)], 17, 3)])
def test_attention_against_a_dense_softmax(sequences, window, sinks):
    batch, cache, q = case(sequences)
    got = attention(batch, cache, q, window=window, sinks=sinks)[0]
    for i, (new, n) in enumerate(sequences):
        j = np.arange(n)
        page, slot = batch.table[i, j // 32], j % 32
        for h in range(4):
            k = torch.from_numpy(fp8.VALUES[cache.k[page, h // 2, slot]] * cache.ks[page, h // 2, slot // 16][:, None])
            v = torch.from_numpy(fp8.VALUES[cache.v[page, h // 2, slot // 16, :, slot % 16]] *
                                 cache.vs[page, h // 2, slot // 16][:, None])
            rows = slice(batch.starts[i], batch.starts[i + 1])
            s = torch.from_numpy(q[rows, h]) @ k.T * 0.125
            p = torch.arange(n - new, n)[:, None] - torch.from_numpy(j)[None]
            hidden = (p < 0) | ((p >= window) & (torch.from_numpy(j)[None] >= sinks) if window else torch.zeros_like(p, dtype=bool))
            want = torch.softmax(s.masked_fill(hidden, -torch.inf), 1) @ v
            assert np.allclose(got[rows, h], want.numpy(), rtol=1e-12, atol=1e-14)


def test_power_scales():
    rng = np.random.default_rng(2)
    for x in np.concatenate([np.exp(rng.uniform(-60, 60, 300)), [448.0, 448.0000001, 447.0, 1.75, 1.0, 2.0 ** -118 * 1.75]]):
        s = fp8_cache.power_scale(x)
        assert x <= 448 * s and (x > 224 * s or s == 2.0 ** -126) and np.log2(s) % 1 == 0
    assert fp8_cache.power_scale(0.0) == fp8_cache.power_scale(1e-40) == 2.0 ** -126


def test_what_is_written_is_near_what_was_given():
    """Half a step of E4M3 of each value, or half of its scale's smallest step; the same where a block is written in
    pieces whose scales grow, with as much again for what was rounded twice."""
    rng = np.random.default_rng(3)
    table = np.array([[1, 0]], dtype=np.int32)
    x = rng.standard_normal((2, 40, 2, 32)) * np.exp(rng.uniform(-4, 2, (2, 40, 1, 1)))
    for pieces in ([40], [1] * 40, [5, 20, 15], [16, 24]):
        cache = random_cache(rng, 2, 2, 32, 32)
        at = 0
        for n in pieces:
            fp8_cache.write(cache, x[0, at:at + n], x[1, at:at + n], [0, n], [at + n], table)
            at += n
        for j in range(40):
            page, block, slot = fp8_cache.place(cache, table, 0, j)
            for h in range(2):
                for codes, scale, want in ((cache.keys(page, h, block), cache.ks[page, h, block], x[0, j, h]),
                                           (cache.values(page, h, block), cache.vs[page, h, block], x[1, j, h])):
                    got = fp8.VALUES[codes[slot]] * scale
                    steps = 2 if len(pieces) > 1 else 1
                    assert (np.abs(got - want) <= steps * np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * scale)).all()


class HostCase(adapters_test.Case):
    def __init__(self, *args):
        adapters_test.gpu, was = (lambda a, dtype=None: torch.as_tensor(a)), adapters_test.gpu
        adapters_test.wide, wide = (lambda t, pad, fill: t), adapters_test.wide
        super().__init__(*args)
        adapters_test.gpu, adapters_test.wide = was, wide

    def exact(self, **change):
        at = lambda name: change.get(name, getattr(self, name))  # noqa: E731
        return fp8.adapters(self.y.double().numpy(), at("codes"), at("scales"), np.asarray(at("down"), dtype=np.float64),
                            np.asarray(at("up"), dtype=np.float64), at("index"), at("factors"))[0]


@pytest.mark.parametrize("kind", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("m,n,k,rank", [(20, 60, 700, 16), (5, 40, 4093, 13), (33, 70, 256, 64)])
def test_right_adapters_pass_and_wrong_ones_do_not(m, n, k, rank, kind):
    c = HostCase(np.random.default_rng([m, n, k]), m, n, k, rank, 4, "bf16", kind)
    c.down, c.up = c.down.double().numpy(), c.up.double().numpy()
    types = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}

    def check(out):
        saved = c.down, c.up
        c.down, c.up = torch.from_numpy(c.down), torch.from_numpy(c.up)
        try:
            c.check(torch.from_numpy(out).to(types[kind]))
        finally:
            c.down, c.up = saved

    check(c.exact())
    wrong = [dict(index=(c.index + 2) % 5 - 1), dict(factors=np.ones(4)), dict(factors=c.factors * 1.02)]
    for name, at in (("down", (slice(None), rank - 1)), ("down", (slice(None), slice(None), slice(k - 64, k))),
                     ("up", (slice(None), slice(None), 0)), ("up", (slice(None), n // 2))):
        lost = np.array(getattr(c, name))
        lost[at] = 0
        wrong.append({name: lost})
    late = c.scales.copy()
    late[:, 1:] = c.scales[:, :-1]
    wrong.append(dict(scales=late))
    for change in wrong:
        with pytest.raises(AssertionError):
            check(c.exact(**change))
