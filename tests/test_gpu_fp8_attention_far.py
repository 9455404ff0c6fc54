"""Attention over the 8-bit cache far from ordinary numbers: scores whose last place is worth more than one, scales at
the ends of 32 bits, positions and windows near 2^31."""
import numpy as np
import pytest
import torch

import cache_bounds
from cache_cases import TYPES, Batch, on_gpu, random_cache
from oracle import fp8, fp8_cache
from paper_2510_23938_amd import hv  # noqa: E402  (a missing library fails the run, never skips it)

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")


def rng_of(*numbers):
    return np.random.default_rng([abs(int(n)) for n in numbers])


def best_keys(cache, q, batch, scale):
    """(value of each row's best key [tokens, heads, dim], by how much its score is ahead, the largest sum of
    |q k| * scale among those that the row sees), in 64 bits."""
    tokens, heads, dim = q.shape
    value, ahead, steep = np.zeros(q.shape), np.full((tokens, heads), np.inf), np.zeros((tokens, heads))
    share = heads // cache.heads
    for i, rows, position in fp8_cache.sequences(batch.starts, batch.lengths, tokens):
        j = np.arange(position + len(rows))
        page, block, slot = np.array([fp8_cache.place(cache, batch.table, i, p) for p in j]).T
        for h in range(heads):
            g = h // share
            keys = fp8.VALUES[cache.k[page, g, block * 16 + slot]] * cache.ks[page, g, block].astype(np.float64)[:, None]
            vals = fp8.VALUES[cache.v[page, g, block, :, slot]] * cache.vs[page, g, block].astype(np.float64)[:, None]
            for n, row in enumerate(rows):
                seen = position + n + 1
                s = keys[:seen] @ q[row, h] * scale
                order = np.argsort(s)
                value[row, h] = vals[order[-1]]
                if seen > 1:
                    ahead[row, h] = s[order[-1]] - s[order[-2]]
                steep[row, h] = (np.abs(keys[:seen]) @ np.abs(q[row, h])).max() * scale
    return value, ahead, steep


# 4, 24 and 160 rows of a sequence's key head: each kernel; the long one is cut into segments
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new,total", [(1, 300), (1, 3000), (6, 300), (40, 300)])
@pytest.mark.parametrize("power", [14, 17, 19, 20, 21, 22, 23, 24, 25, 26, 27, 28, 30, 40, 64, 100])
def test_large_scores(new, total, dtype, power):
    """Finite scores of up to about 2^(power + 5): where the best key's is ahead by more than 100 and what 32 bits lose
    (the bound of cache_bounds.py, and the product's and the subtraction's last places), its value is the output, up to the
    roundings of its weight and of the result.  Every output is finite and no larger than the values."""
    rng = rng_of(power, new, total)
    batch = Batch(rng, [(new, total), (new, new), (1, 1), (new, new + 20)], 32)
    host = random_cache(rng, batch.pool, 2, 32, 64)
    host.ks *= np.float32(2.0 ** power)
    q = torch.from_numpy(rng.standard_normal((batch.tokens, 8, 64))).to(TYPES[dtype])
    out = hv.hv_fp8_attention(q.to(DEV), on_gpu(host), *batch.gpu()).double().cpu().numpy()
    value, ahead, steep = best_keys(host, q.double().numpy(), batch, 0.125)
    assert np.isfinite(out).all()
    largest = np.abs(fp8.VALUES[host.v[np.isin(np.arange(host.pages), batch.table)] & 0x7f]).max() * host.vs.max()
    assert (np.abs(out) <= largest).all()
    clear = ahead > 100 + (200 * 2.0 ** -24 + 2.0 ** -21) * steep
    assert clear.mean() > 0.5
    half = cache_bounds.HALF_STEP[dtype]
    off = np.abs(out - value)
    assert (off[clear] <= (2 * half + 2.0 ** -20) * np.abs(value[clear]) + (2.0 ** -25 if dtype == "f16" else 2.0 ** -134)).all()


@pytest.mark.parametrize("new", [1, 6, 40])
def test_small_key_scales_under_large_queries(new):
    """Key scales of 2^-126 times the softmax's scale are below the smallest normal number; queries of 2^115 make scores
    of ordinary size of them."""
    rng = rng_of(new)
    batch = Batch(rng, [(new, 300), (new, 41)], 32)
    host = random_cache(rng, batch.pool, 2, 32, 64)
    host.ks[:] = 2.0 ** -126
    q = torch.from_numpy(rng.standard_normal((batch.tokens, 8, 64)) * 2.0 ** 115).to(torch.bfloat16)
    out = hv.hv_fp8_attention(q.to(DEV), on_gpu(host), *batch.gpu())
    want = fp8_cache.attention(host, q.double().numpy(), batch.starts, batch.lengths, batch.table, 0.125)
    cache_bounds.check(out.double().cpu().numpy(), want, "bf16", 300)


@pytest.mark.parametrize("new", [1, 6, 40])
@pytest.mark.parametrize("length,window,same_length,same_window", [
    ((1 << 31) - 1, 0, 1000, 0), ((1 << 31) - 1, (1 << 31) - 1, 1000, 0), ((1 << 31) - 1, 1 << 31, 1000, 0),
    ((1 << 31) - 1, (1 << 32) - 1, 1000, 0), ((1 << 30) + 300, (1 << 30) + 200, 300, 200), (250, (1 << 31) - 1, 250, 0),
    ((1 << 31) - 1, (1 << 31) - 1 - 150, 300, 150), (3, (1 << 31) - 1, 3, 0), (3, (1 << 30) + 5, 3, 0)])
def test_far_positions(new, length, window, same_length, same_window):
    """Tokens behind the table's last column see what is in the cache: as much as nearer ones with a window that reaches
    as far, bit for bit.  Tokens ahead of the first see nothing."""
    rng = rng_of(new, length, window)
    batch = Batch(rng, [(new, 240)], 48)
    host = on_gpu(random_cache(rng, batch.pool, 2, 48, 64))
    starts, _, table = batch.gpu()
    q = torch.from_numpy(rng.standard_normal((new, 8, 64))).to(torch.bfloat16).to(DEV)
    far, near = (hv.hv_fp8_attention(q, host, starts, torch.tensor([n], dtype=torch.int32, device=DEV), table, window=w)
                 for n, w in ((length, window), (same_length, same_window)))
    assert bool(near[-1].any())
    assert torch.equal(far.view(torch.int16), near.view(torch.int16))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new", [1, 3, 20])
def test_many_sequences(dtype, new):
    """More than ten times as many as a wave looks at at once, short ones and a few that are cut."""
    rng = rng_of(new, 700)
    lengths = rng.integers(0, 60, 700)
    lengths[[5, 300, 301, 650, 699]] = [2500, 1800, 4000, 3000, 1700]
    batch = Batch(rng, [(min(int(rng.integers(0, new + 1)) if n < 100 else new, int(n)), int(n)) for n in lengths], 16)
    host = random_cache(rng, batch.pool, 1, 16, 32)
    q = torch.from_numpy(rng.standard_normal((batch.tokens, 4, 32))).to(TYPES[dtype])
    out = hv.hv_fp8_attention(q.to(DEV), on_gpu(host), *batch.gpu())
    want = fp8_cache.attention(host, q.double().numpy(), batch.starts, batch.lengths, batch.table, 32 ** -0.5)
    cache_bounds.check(out.double().cpu().numpy(), want, dtype, 60)


@pytest.mark.parametrize("new", [1, 6, 40])
def test_values_near_the_smallest_numbers(new):
    """Values under a scale of 2^-126, in units of it; half of the dimensions have values below it.  bfloat16 holds those as
    multiples of 2^-7 units, and codes are multiples of 2^-9: a value is off by up to 2^-8 units, their mean by weights that
    add up to one by as much, and the result's rounding by as much again."""
    rng = rng_of(new, 4)
    batch = Batch(rng, [(new, 300), (new, 41)], 32)
    host = random_cache(rng, batch.pool, 2, 32, 64)
    host.vs[:] = 2.0 ** -126
    host.v[:, :, :, ::2] = fp8.round_to_code(rng.uniform(-2, 2, host.v[:, :, :, ::2].shape))
    q = torch.from_numpy(rng.standard_normal((batch.tokens, 8, 64))).to(torch.bfloat16)
    out = hv.hv_fp8_attention(q.to(DEV), on_gpu(host), *batch.gpu()).double().cpu().numpy() * 2.0 ** 126
    units = host.copy()
    units.vs[:] = 1.0
    want, size, root, steep = fp8_cache.attention(units, q.double().numpy(), batch.starts, batch.lengths, batch.table, 0.125)
    half = cache_bounds.HALF_STEP["bf16"]
    weights = 2 * (100 * 2.0 ** -24 * steep + 2.0 ** -21 + 2.0 ** -18)[:, :, None]
    allowed = weights * size + 6 * half / np.sqrt(3) * root + half * np.abs(want) + 2 * 2.0 ** -8
    assert (np.abs(out - want) <= allowed).all()


@pytest.mark.parametrize("new", [1, 6, 40])
def test_offsets_past_32_bits(new):
    """Pages behind the first 4 GiB of a pool, and tokens' rows behind the first 4 GiB of queries and outputs."""
    rng = rng_of(new, 32)
    batch = Batch(rng, [(new, 300)], 32, spare=2)
    host = random_cache(rng, batch.pool, 2, 32, 64)
    apart, far = 1 << 29, 1 << 26 if new > 1 else 128
    codes = []
    for a in (host.k, host.v):
        raw = torch.empty(batch.pool * apart, dtype=torch.uint8, device=DEV)
        inner = (64, 1) if a.ndim == 4 else (1024, 16, 1)
        t = raw.as_strided(a.shape, (apart, 2048, *inner))
        t.copy_(torch.from_numpy(a).to(DEV))
        codes.append(t.view(torch.float8_e4m3fn))
    assert int(batch.table.max()) * apart > 1 << 32
    cache = hv.Fp8Cache(codes[0], torch.from_numpy(host.ks).to(DEV), codes[1], torch.from_numpy(host.vs).to(DEV))
    rows = [torch.empty(far * new, dtype=torch.bfloat16, device=DEV).as_strided((new, 8, 64), (far, 64, 1)) if far > 128 else
            torch.empty(new, 8, 64, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    q = torch.from_numpy(rng.standard_normal((new, 8, 64))).to(torch.bfloat16)
    rows[0].copy_(q.to(DEV))
    hv.hv_fp8_attention(rows[0], cache, *batch.gpu(), out=rows[1])
    want = fp8_cache.attention(host, q.double().numpy(), batch.starts, batch.lengths, batch.table, 0.125)
    cache_bounds.check(rows[1].double().cpu().numpy(), want, "bf16", 300)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("new", [1, 12, 40])
def test_a_very_long_context(dtype, new):
    """Three million tokens, against a softmax in 64 bits on the GPU."""
    gen = torch.Generator(device=DEV).manual_seed(new)
    length, page, dim = 3_000_001, 1024, 16
    pages = -(-length // page)
    cache = hv.Fp8Cache.empty(pages, 1, page, dim, DEV)
    for t in (cache.k_codes, cache.v_codes):
        t.copy_((torch.randn(t.shape, generator=gen, device=DEV) * 30).to(t.dtype))
    cache.k_scales.fill_(2.0 ** -5)
    cache.v_scales.copy_(torch.exp2(torch.randint(-6, 1, cache.v_scales.shape, generator=gen, device=DEV).float()))
    table = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32).view(1, pages)
    q = torch.randn(new, 2, dim, generator=gen, device=DEV).to(TYPES[dtype])
    starts, lengths = (torch.tensor(a, dtype=torch.int32, device=DEV) for a in ([0, new], [length]))
    out = hv.hv_fp8_attention(q, cache, starts, lengths, table).double()
    order = table[0].long()
    k = cache.k_codes[order].float().double().view(-1, dim) * 2.0 ** -5
    v = cache.v_codes[order].float().double() * cache.v_scales[order].double()[..., None, None]
    v = v.transpose(3, 4).reshape(-1, dim)
    half = cache_bounds.HALF_STEP[dtype]
    for n in range(new):
        seen = length - new + n + 1
        for h in range(2):
            s = (k[:seen] * q[n, h].double()).sum(1) * 0.25
            w = torch.softmax(s, 0)[:, None]
            want, size = (w * v[:seen]).sum(0), (w * v[:seen].abs()).sum(0)
            root = ((w * v[:seen]) ** 2).sum(0).sqrt()
            steep = float((k[:seen].abs() * q[n, h].double().abs()).sum(1).max()) * 0.25
            allowed = 2 * (100 * 2.0 ** -24 * steep + 2.0 ** -21 + 2.0 ** -18) * size + 6 * half / 3 ** 0.5 * root + half * want.abs()
            if dtype == "f16":  # weights that are subnormal numbers (half_bounds.py), and a subnormal result
                p = torch.exp(s - s.max()) * cache.v_scales[order].double().view(-1, 1).expand(-1, 16).reshape(-1)[:seen] * 16
                small = p < 2.0 ** -14
                codes = (v[:seen] / cache.v_scales[order].double().view(-1, 1).expand(-1, 16).reshape(-1, 1)[:seen]).abs()
                lost = (torch.clamp(p, max=2.0 ** -25) * small)[:, None] * codes
                allowed += lost.sum(0) / 16 / torch.exp(s - s.max()).sum() + 2.0 ** -25
            assert bool(((out[n, h] - want).abs() <= allowed).all()), (n, h, ((out[n, h] - want).abs() / allowed).max())
