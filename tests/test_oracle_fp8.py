"""The 8-bit oracle against what it is not made from: torch's own E4M3 type and brute force."""
import numpy as np
import pytest
import torch

from oracle import fp8


def test_values_are_the_formats():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(fp8.VALUES, want, equal_nan=True)
    assert np.nanmax(fp8.VALUES) == fp8.LARGEST and np.isnan(fp8.VALUES[[0x7f, 0xff]]).all()


def test_rounding_every_neighbourhood():
    v = fp8.VALUES[:127]
    mid = (v[:-1] + v[1:]) / 2
    points = np.concatenate([v, mid, np.nextafter(mid, 0), np.nextafter(mid, 1e9), [463.9, 448.1]])
    points = np.concatenate([points, -points]).astype(np.float32)
    want = torch.from_numpy(points).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(fp8.round_to_code(points), want)
    assert fp8.round_to_code([np.nan, np.inf, -np.inf]).tolist()[0] & 0x7f == 0x7f
    assert (fp8.round_to_code([np.inf, -np.inf]) & 0x7f == 0x7f).all()


def test_rounding_is_nearest():
    rng = np.random.default_rng(5)
    q = rng.standard_normal(4000) * np.exp(rng.uniform(-8, 5, 4000))
    q = np.clip(q, -448, 448)
    got = fp8.VALUES[fp8.round_to_code(q)]
    best = np.nanmin(np.abs(fp8.VALUES[None, :] - q[:, None]), 1)
    assert np.array_equal(np.abs(got - q), best)


@pytest.mark.parametrize("tile", [1, 128])
def test_group_scales(tile):
    rng = np.random.default_rng(6)
    y = rng.standard_normal((130, 259))
    y[3, 5], y[3, 6] = np.inf, np.nan
    y[129] = 0
    s = fp8.group_scales(y, tile)
    assert s.shape == (130 if tile == 1 else 2, 3)
    if tile == 1:
        assert (s[129] == 1).all()
        assert s[3, 0] == np.float32(np.abs(np.delete(y[3, :128], [5, 6])).max() / 448)
        assert s[7, 2] == np.float32(np.abs(y[7, 256:]).max() / 448)
    else:
        assert s[1, 1] == np.float32(np.abs(y[128:, 128:256]).max() / 448)
    e = fp8.spread(s, tile, *y.shape)
    assert e.shape == y.shape and e[128, 258] == s[128 // tile, 2]


def test_matmul_by_hand():
    rng = np.random.default_rng(7)
    a, b = rng.integers(0, 127, (3, 200)).astype(np.uint8), rng.integers(0, 127, (131, 200)).astype(np.uint8)
    sa, sb = rng.random((3, 2)), rng.random((2, 2))
    c, size = fp8.matmul(a, sa, b, sb)
    for i, j in ((0, 0), (2, 130), (1, 127)):
        want = sum(fp8.VALUES[a[i, t]] * sa[i, t // 128] * fp8.VALUES[b[j, t]] * sb[j // 128, t // 128]
                   for t in range(200))
        assert abs(c[i, j] - want) <= 1e-12 * size[i, j]


def test_norm_and_gated():
    x = np.array([[3.0, 4.0]])
    y, h = fp8.rms_norm(x, None, np.ones(2), 0.0)
    assert np.allclose(y, x / np.sqrt(12.5)) and np.array_equal(h, x)
    y, h = fp8.rms_norm(x, x, np.array([1.0, 2.0]), 1.0)
    assert np.allclose(y, [[6 / np.sqrt(51), 16 / np.sqrt(51)]]) and np.array_equal(h, 2 * x)
    assert np.allclose(fp8.gated([[0.0, 1.0, -1000.0]], [[5.0, 2.0, 3.0]]), [[0, 2 / (1 + np.exp(-1)), 0]])
