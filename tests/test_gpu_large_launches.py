"""Calls of more items than one row of a launch holds (2^20): the launch's last row is filled up with workgroups past the
last item.  All values are small whole numbers, so that results are exact in any order."""
import pytest
import torch

from paper_2510_23938_amd import hv  # noqa: E402  (a missing library fails the run, never skips it)

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
E4M3 = torch.float8_e4m3fn


def whole(gen, low, high, *shape, dtype=torch.bfloat16):
    return torch.randint(low, high + 1, shape, generator=gen, dtype=torch.int8, device=DEV).to(dtype)


# a workgroup takes 64 columns of one tile of 16 tokens, or 128 of four tiles: 2^20 + 1 items, 2^20 + 59, 2^20 + 1
@pytest.mark.parametrize("m,n", [(16, (1 << 26) + 1), (1000, 16645 * 64 - 3), ((1 << 26) + 1, 1)])
def test_adapters(m, n):
    gen = torch.Generator(device=DEV).manual_seed(m)
    x = whole(gen, 0, 1, m, 1, dtype=torch.float32).to(E4M3)
    y = whole(gen, -8, 8, m, n)
    down, up = whole(gen, -1, 1, 2, 1, 1), whole(gen, -2, 2, 2, n, 1)
    index = whole(gen, -1, 1, m, dtype=torch.int32)
    want = y.clone()
    mine = index.long().clamp_min(0)
    inner = torch.where(index >= 0, x.float()[:, 0] * down.float()[mine, 0, 0], 0.0).to(torch.bfloat16)
    if n == 1:
        want += inner[:, None] * up[mine, :, 0]
    else:
        for t in range(m):
            want[t] += inner[t] * up[int(mine[t]), :, 0]
    hv.hv_fp8_adapters(y, x, torch.ones(m, 1, device=DEV), down, up, index, out=y)
    assert torch.equal(y, want)


def test_cache_write():
    """A sequence of 2^24 tokens less three, from the middle of a block: 2^20 blocks, and room for two more."""
    gen = torch.Generator(device=DEV).manual_seed(1)
    tokens, page = (1 << 24) - 3, 65536
    cache = hv.Fp8Cache.empty(257, 1, page, 16, DEV)
    k, v = (whole(gen, -15, 15, tokens, 1, 16, dtype=torch.float16) for _ in range(2))
    pages = torch.arange(256, -1, -1, dtype=torch.int32, device=DEV).view(1, 257)
    first = 5
    batch = [torch.tensor(a, dtype=torch.int32, device=DEV) for a in ([0, tokens], [tokens + first])]
    hv.hv_fp8_cache_write(cache, k, v, *batch, pages)
    codes = cache.k_codes.to(torch.float16).view(257, -1, 16, 16).flip(0) * cache.k_scales.half().view(257, -1, 1, 1).flip(0)
    assert torch.equal(codes.view(-1, 16)[first:first + tokens], k[:, 0])
    codes = cache.v_codes.to(torch.float16).view(257, -1, 16, 16).flip(0) * cache.v_scales.half().view(257, -1, 1, 1).flip(0)
    assert torch.equal(codes.transpose(2, 3).reshape(-1, 16)[first:first + tokens], v[:, 0])
    assert bool((cache.k_codes.view(torch.uint8).view(257, -1)[0, 16 * (first + 10):] == 0).all())


@pytest.mark.parametrize("new", [1, 32, 40])
def test_attention(new):
    """A key head's values of a sequence are all the same, so each output is that value, up to a weight's rounding and
    the result's: 1000 sequences of 1100 key heads."""
    gen = torch.Generator(device=DEV).manual_seed(new)
    count, heads, dim = 1000, 1100, 16
    cache = hv.Fp8Cache.empty(3 * count, heads, 16, dim, DEV)
    cache.k_codes.copy_(whole(gen, -3, 3, 3 * count, heads, 16, dim, dtype=torch.float16).to(E4M3))
    value = whole(gen, -15, 15, count, heads, 1, 1, 1, dtype=torch.float16)
    cache.v_codes.copy_(value.repeat_interleave(3, 0).expand(-1, -1, 1, dim, 16).to(E4M3))
    cache.k_scales.fill_(1.0)
    cache.v_scales.fill_(0.5)
    q = torch.randn(count * new, heads, dim, generator=gen, device=DEV, dtype=torch.bfloat16)
    batch = [torch.arange(count + 1, dtype=torch.int32, device=DEV) * new,
             torch.full((count,), 41, dtype=torch.int32, device=DEV),
             torch.arange(3 * count, dtype=torch.int32, device=DEV).view(count, 3)]
    out = hv.hv_fp8_attention(q, cache, *batch).float()
    want = (value.float() * 0.5).view(count, 1, heads, 1)
    off = (out.view(count, new, heads, dim) - want).abs()
    assert bool((off <= 2.0 ** -7 * want.abs()).all())
