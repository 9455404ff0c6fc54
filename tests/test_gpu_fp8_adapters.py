"""Adapters beside a product against their definition in 64 bits (oracle/fp8.py).

Products of codes and 16-bit weights are exact in 32 bits.  A term of the inner row passes up to 128 additions within a
group, one for each group, 4 + 16 where waves' and parts' sums meet, and as part of the second product up to 1024 / 4;
each rounds by up to 2^-24 of a partial sum, which the terms' magnitudes' sum bounds, with a sign of its own: six
standard deviations of their number, and 8 more of them for the scales' and factors' products.  The result is rounded once."""
import numpy as np
import pytest
import torch

from oracle import fp8
from paper_2510_23938_amd import hv  # noqa: E402  (a missing library fails the run, never skips it)

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


def gpu(a, dtype=None):
    t = torch.as_tensor(a)
    return (t if dtype is None else t.to(dtype)).to(DEV)


def wide(t, pad, fill):
    """The same matrix with ``pad`` elements of ``fill`` between its rows."""
    if t.dtype == torch.float8_e4m3fn:
        return wide(t.view(torch.uint8), pad, fill).view(torch.float8_e4m3fn)
    w = torch.full((t.shape[0], t.shape[1] + pad), fill, dtype=t.dtype, device=DEV)
    w[:, :t.shape[1]] = t
    return w[:, :t.shape[1]]


class Case:
    def __init__(self, rng, m, n, k, rank, adapters, dtype, kind, index=None, pad=0):
        self.kind = kind
        x = fp8.round_to_code(np.clip(rng.standard_normal((m, k)) * 60, -448, 448))
        self.scales = np.exp2(rng.uniform(-8, -6, (m, -(-k // 128)))).astype(np.float32)
        self.down = torch.from_numpy(rng.standard_normal((adapters, rank, k)) * (k + 1) ** -0.5).to(TYPES[dtype])
        self.up = torch.from_numpy(rng.standard_normal((adapters, n, rank))).to(TYPES[dtype])
        self.factors = rng.uniform(0.5, 2, adapters).astype(np.float32)
        self.index = (rng.integers(-1, adapters, m) if index is None else np.asarray(index)).astype(np.int32)
        self.y = torch.from_numpy(rng.standard_normal((m, n))).to(TYPES[kind])
        self.codes = x
        self.args = [wide(gpu(self.y), pad, float("nan")), wide(gpu(x).view(torch.float8_e4m3fn), pad, 0x7f),
                     gpu(self.scales), gpu(self.down), gpu(self.up), gpu(self.index), gpu(self.factors)]

    def check(self, got, factors=None):
        want, size = fp8.adapters(self.y.double().numpy(), self.codes, self.scales, self.down.double().numpy(),
                                  self.up.double().numpy(), self.index, self.factors if factors is None else factors)
        m, k = self.codes.shape
        additions = 128 + -(-k // 128) + 20 + self.down.shape[1] / 4
        allowed = (6 * np.sqrt(additions) + 8) * 2.0 ** -24 * size + HALF_STEP[self.kind] * np.abs(want)
        off = np.abs(got.double().cpu().numpy() - want)
        assert (off <= allowed).all(), (np.argwhere(~(off <= allowed))[:5], np.nanmax(off / allowed))


def check(rng, m, n, k, rank, adapters, dtype="bf16", kind="bf16", index=None, pad=0):
    c = Case(rng, m, n, k, rank, adapters, dtype, kind, index, pad)
    raw = torch.full((m + 2, n + pad), 7.0, dtype=TYPES[kind], device=DEV)
    out = raw[1:-1, :n]
    ws = hv.Workspace(DEV)
    assert hv.hv_fp8_adapters(*c.args, out=out, workspace=ws) is out
    c.check(out)
    frame = raw.clone()
    frame[1:-1, :n] = 7.0
    assert bool((frame == 7.0).all())
    assert torch.equal(hv.hv_fp8_adapters(*c.args, workspace=ws), out)
    return c, out


def rng_of(*numbers):
    return np.random.default_rng(list(numbers))


@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 40, 130])
@pytest.mark.parametrize("n,k", [(1, 1), (64, 128), (65, 100), (1000, 16), (200, 4093), (16, 2048), (130, 1000)])
def test_sizes(m, n, k):
    check(rng_of(m, n, k), m, n, k, 16, 5)
    check(rng_of(m, n, k, 1), m, n, k, 8, 3, "f16", "f32", pad=3)


@pytest.mark.parametrize("rank", [1, 2, 3, 4, 7, 13, 16, 17, 32, 60, 64, 65, 100, 128, 130, 1024])
def test_ranks(rank):
    check(rng_of(rank), 20, 100, 700, rank, 3)
    check(rng_of(rank, 1), 5, 70, 300, rank, 2, "f16", "f16", pad=1)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_types(dtype, kind):
    check(rng_of(1), 50, 300, 900, 16, 4, dtype, kind)
    check(rng_of(2), 50, 301, 901, 12, 4, dtype, kind, pad=5)


@pytest.mark.parametrize("index", [[0] * 40, [-1] * 40, list(range(40)), [3] * 7 + [-1] + [39] * 32, [40, 1 << 30, -5] + [2] * 37,
                                   [0, 1] * 20, [5] * 16 + [6] * 24], ids=lambda i: str(i[:9]))
def test_orders(index):
    """One adapter for all, none, another for each token, numbers of no adapter."""
    check(rng_of(3), 40, 200, 500, 16, 40, index=index)


def test_many_tokens():
    """More than a workgroup's tokens of the second kernel, prompts of different lengths."""
    rng = rng_of(4)
    index = np.repeat(np.arange(9) % 4 - 1, rng.integers(1, 400, 9))[:1500]
    check(rng, len(index), 130, 300, 16, 3, index=index)
    check(rng, len(index), 65, 200, 40, 3, "f16", "f32", index=index)


def test_in_place_and_without_factors():
    rng = rng_of(5)
    c = Case(rng, 30, 257, 500, 16, 4, "bf16", "bf16")
    y, rest = c.args[0].clone(), c.args[1:]
    assert hv.hv_fp8_adapters(y, *rest, out=y) is y
    c.check(y)
    c.check(hv.hv_fp8_adapters(*c.args[:-1]), np.ones(4))


def test_leading_dimensions_of_tokens():
    rng = rng_of(6)
    c = Case(rng, 24, 100, 256, 8, 3, "bf16", "bf16")
    y, x, s, down, up, index, factors = c.args
    out = hv.hv_fp8_adapters(y.view(2, 12, 100), x.view(2, 12, 256), s.view(2, 12, 2), down, up, index.view(2, 12), factors)
    c.check(out.view(24, 100))


def test_no_adapters_and_nothing_to_write():
    rng = rng_of(7)
    c = Case(rng, 5, 70, 130, 4, 2, "bf16", "bf16")
    y, x, s, down, up, index, factors = c.args
    assert torch.equal(hv.hv_fp8_adapters(y, x, s, down[:0], up[:0], index, factors[:0]), y)
    none = hv.hv_fp8_adapters(y, x[:, :0], s[:, :0], down[:, :, :0].contiguous(), up, index, factors)
    assert torch.equal(none, y)
    assert hv.hv_fp8_adapters(y[:0], x[:0], s[:0], down, up, index[:0], factors).shape == (0, 70)
    assert hv.hv_fp8_adapters(y[:, :0], x, s, down, up[:, :0], index, factors).shape == (5, 0)


def test_a_tokens_output_is_its_own():
    """NaN and infinities in one adapter, one token's codes and scales reach that adapter's and that token's outputs alone."""
    rng = rng_of(8)
    c = Case(rng, 40, 90, 300, 16, 4, "bf16", "bf16", index=[0, 1, 2, 3] * 10)
    good = hv.hv_fp8_adapters(*c.args)
    y, x, s, down, up, index, factors = c.args
    down, up, x, s = down.clone(), up.clone(), x.clone(), s.clone()
    down[1, 3, 7], up[2, 5, 2] = float("inf"), float("nan")
    x.view(torch.uint8)[4, 9] = 0x7f
    s[8, 1] = float("nan")
    out = hv.hv_fp8_adapters(y, x, s, down, up, index, factors)
    same = torch.ones(40, 90, dtype=torch.bool, device=DEV)
    same[1::4] = False
    same[2::4, 5] = False
    same[4] = same[8] = False
    assert torch.equal(out[same], good[same])
    assert bool(torch.isnan(out[2::4, 5]).all()) and bool(torch.isnan(out[4]).all()) and bool(torch.isnan(out[8]).all())
    assert not bool(torch.isfinite(out[1::4]).any())


def test_offsets_past_32_bits():
    """An adapter whose weights lie behind the first 4 GiB."""
    rng = rng_of(9)
    rank, k, n, adapters = 16, 8192, 24, 17000
    down = torch.zeros(adapters, rank, k, dtype=torch.bfloat16, device=DEV)
    up = torch.zeros(adapters, n, rank, dtype=torch.bfloat16, device=DEV)
    c = Case(rng, 5, n, k, rank, 1, "bf16", "f32", index=[0] * 5)
    down[-1], up[-1] = c.args[3][0], c.args[4][0]
    index = torch.full((5,), adapters - 1, dtype=torch.int32, device=DEV)
    out = hv.hv_fp8_adapters(*c.args[:3], down, up, index, c.args[6].expand(adapters).contiguous())
    c.check(out)


@pytest.mark.parametrize("m", [1, 40, 1100])
@pytest.mark.parametrize("kind", TYPES)
def test_tokens_without_an_adapter_keep_their_bits(m, kind):
    """Zeros of either sign, the smallest numbers, infinities and NaN among them: out[t] is y[t]."""
    rng = rng_of(m)
    c = Case(rng, m, 90, 300, 16, 3, "bf16", kind, index=np.where(np.arange(m) % 3 == 0, -1, np.arange(m) % 3))
    y, x, s, down, up, index, factors = c.args
    tiny = torch.finfo(y.dtype).smallest_normal
    special = torch.tensor([0.0, -0.0, tiny / 4, -tiny / 4, float("inf"), -float("inf"), 1.0], device=DEV).to(y.dtype)
    y[:, ::2] = special.repeat(7)[:45]
    bits = {2: torch.int16, 4: torch.int32}[y.element_size()]
    none = index < 0
    for args in ((y, x, s, down, up, index, factors), (y, x, s, down[:0], up[:0], index, factors[:0]),
                 (y, x[:, :0], s[:, :0], down[:, :, :0].contiguous(), up, index, factors)):
        out = hv.hv_fp8_adapters(*args)
        kept = none if args[3].numel() else torch.ones_like(none)
        assert torch.equal(out[kept].view(bits), y[kept].view(bits))
