"""The 8-bit operators (hv_fp8.h) against their definitions in 64 bits (oracle/fp8.py).

What is allowed, from the operators' arithmetic:

* scales: a quantised matrix's are exact (one rounding of max / 448); behind the
  norm and the gate they move with y, whose relative error is below ``Y_ERROR``;
* codes: equal to the quotient's rounding, or to that of a quotient within the
  arithmetic's relative error of it (``Q_ERROR`` for the quotient alone: the scale's
  reciprocal and the product round once each);
* products: every term is exact in 32 bits; a sum over k terms and its groups
  moves by at most 2^-23 per addition of the terms' magnitudes' sum, and the result
  rounds once to its type.  For the 16-bit types the matrix unit adds 16
  products in fixed point, down to 2^-13 of the largest: codes whose exponents lie within
  4 binades lose nothing there (products span 2^10 to 2^17.7 in steps of 2^4), other codes up to
  15 * 2^-13 of the terms' magnitudes.
"""
import numpy as np
import pytest
import torch

from oracle import fp8
from paper_2510_23938_amd import hv  # noqa: E402  (a missing library fails the run, never skips it)

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
HALF_ULP = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}
Q_ERROR = 2.0 ** -22
Y_ERROR = 2.0 ** -17
CANARY = 0x55


def values(rng, shape, kind="normal"):
    x = rng.standard_normal(shape)
    if kind == "spread":  # magnitudes over many binades, some zeros
        x = x * np.exp(rng.uniform(-12, 6, shape)) * (rng.random(shape) > 0.1)
    return x


def on_gpu(x, dtype, pad=0, offset=0):
    """x on the GPU in a wider matrix, ``pad`` elements between rows, its first element ``offset`` elements
    into the allocation; what lies between is NaN."""
    x = torch.as_tensor(x).to(dtype)
    rows, cols = x.shape
    flat = torch.full((offset + rows * (cols + pad),), float("nan"), dtype=torch.float32).to(dtype).to(DEV)
    wide = flat[offset:].view(rows, cols + pad)
    t = wide[:, :cols]
    t.copy_(x.to(DEV))
    return t


def codes_on_gpu(codes, pad=0, offset=0):
    rows, cols = codes.shape
    flat = torch.full((offset + rows * (cols + pad),), 0x7f, dtype=torch.uint8, device=DEV)
    t = flat[offset:].view(rows, cols + pad)[:, :cols]
    t.copy_(torch.from_numpy(codes).to(DEV))
    return t.view(torch.float8_e4m3fn)


def framed(rows, cols, dtype, pad, fill=CANARY):
    """([rows, cols] view, whole byte buffer): an output with canaries before, between and after its rows."""
    size = torch.empty((), dtype=dtype).element_size()
    raw = torch.full((64 + rows * (cols + pad) * size + 64,), fill, dtype=torch.uint8, device=DEV)
    return raw[64:-64].view(dtype).view(rows, cols + pad)[:, :cols], raw


def frame_untouched(raw, rows, cols, pad, size, fill=CANARY):
    b = raw.cpu().numpy()
    inner = b[64:-64].reshape(rows, (cols + pad) * size)
    return (b[:64] == fill).all() and (b[-64:] == fill).all() and (inner[:, cols * size:] == fill).all()


def bytes_of(t):
    return t.contiguous().view(torch.uint8).cpu().numpy()


def check_codes(got, y, scales, tile_rows, error):
    q = y / fp8.spread(scales, tile_rows, *y.shape)
    low, high = fp8.round_to_code(q * (1 - error)), fp8.round_to_code(q * (1 + error))
    nan = ~np.isfinite(y)
    assert ((got[nan] & 0x7f) == 0x7f).all()
    same = (got == low) | (got == high)
    zero = (fp8.VALUES[low] == 0) & (fp8.VALUES[got] == 0)  # a zero's sign is free where it rounds to zero
    assert (same | zero | nan).all(), np.argwhere(~(same | zero | nan))[:5]


# --------------------------------------------------------------------------
# quantisation

SHAPES = [(1, 1), (1, 128), (3, 7), (5, 129), (16, 1024), (127, 255), (128, 128), (129, 257), (300, 136), (2, 5000),
          (257, 2048), (1, 40000)]


@pytest.mark.parametrize("tile", ["rows", "blocks"])
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", TYPES)
def test_quantize(tile, rows, cols, dtype):
    rng = np.random.default_rng([rows, cols, 1])
    for pad, offset, kind in ((0, 0, "normal"), (3, 1, "spread"), (8, 0, "spread")):
        x = on_gpu(values(rng, (rows, cols), kind), TYPES[dtype], pad, offset)
        out, raw = framed(rows, cols, torch.float8_e4m3fn, pad)
        codes, scales = hv.hv_fp8_quantize(x, tile, out=out)
        y = x.double().cpu().numpy()
        t = 1 if tile == "rows" else 128
        assert np.array_equal(scales.cpu().numpy(), fp8.group_scales(y, t))
        check_codes(bytes_of(codes), y, scales.cpu().numpy(), t, Q_ERROR)
        assert frame_untouched(raw, rows, cols, pad, 1)


@pytest.mark.parametrize("tile", ["rows", "blocks"])
@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_special_values(tile, dtype):
    x = np.zeros((130, 300))
    x[0, :5] = [np.nan, np.inf, -np.inf, 1.0, -2.0]
    x[1, 128:256] = np.nan
    x[129, 290] = np.finfo(np.float32).max if dtype != "f16" else 65504
    x[2, 10:14] = [1e-38, -1e-40, 1e-45, 0] if dtype != "f16" else [6e-8, -6e-8, 1e-5, 0]
    x = on_gpu(x, TYPES[dtype])
    codes, scales = hv.hv_fp8_quantize(x, tile)
    y = x.double().cpu().numpy()
    t = 1 if tile == "rows" else 128
    assert np.array_equal(scales.cpu().numpy(), fp8.group_scales(y, t))
    check_codes(bytes_of(codes), y, scales.cpu().numpy(), t, Q_ERROR)


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_divides(dtype):
    """The codes of the rounded quotient, ties among them (frequent for 16-bit values), for scales of many binades."""
    rng = np.random.default_rng(15)
    x = on_gpu(values(rng, (512, 1024)) * np.exp(rng.uniform(-60, 60, (512, 1)) if dtype != "f16" else 0), TYPES[dtype])
    codes, scales = hv.hv_fp8_quantize(x)
    quotient = x.float().cpu().numpy() / np.repeat(scales.cpu().numpy(), 128, 1)
    assert quotient.dtype == np.float32
    assert np.array_equal(bytes_of(codes), fp8.round_to_code(quotient))


def test_quantize_keeps_ties_to_even():
    # every midpoint of neighbouring codes under a scale of one: exact quotients
    v = fp8.VALUES[:127]
    x = np.concatenate([v, (v[:-1] + v[1:]) / 2, [448.0]])
    x = np.concatenate([x, -x])[:, None] * np.ones((1, 128))
    x[:, 1] = 448.0  # the group's largest: a scale of one
    codes, scales = hv.hv_fp8_quantize(on_gpu(x, torch.float32))
    assert (scales == 1).all()
    assert np.array_equal(bytes_of(codes), fp8.round_to_code(x))


# --------------------------------------------------------------------------
# norm

@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows,cols", SHAPES + [(3, 8192), (2, 16392), (2, 33000), (700, 64)])
@pytest.mark.parametrize("dtype", TYPES)
def test_rms_norm(residual, rows, cols, dtype):
    rng = np.random.default_rng([rows, cols, 2])
    for pad, offset in ((0, 0), (5, 1)):
        x = on_gpu(values(rng, (rows, cols)), TYPES[dtype], pad, offset)
        r = on_gpu(values(rng, (rows, cols)), TYPES[dtype], pad) if residual else None
        w = torch.from_numpy(1 + 0.3 * rng.standard_normal(cols)).to(TYPES[dtype]).to(DEV)
        out, raw = framed(rows, cols, torch.float8_e4m3fn, pad)
        h, raw_h = framed(rows, cols, TYPES[dtype], pad)
        codes, scales, h = hv.hv_fp8_rms_norm(x, w, 1e-5, residual=r, out=out, residual_out=h if residual else None)
        y, want_h = fp8.rms_norm(x.float().cpu().numpy(), r.float().cpu().numpy() if residual else None,
                                 w.double().cpu().numpy(), np.float32(1e-5))
        got = scales.cpu().numpy()
        assert np.all(np.abs(got / fp8.group_scales(y, 1) - 1) <= Y_ERROR)
        check_codes(bytes_of(codes), y, got, 1, 2 * Y_ERROR)
        size = torch.empty((), dtype=TYPES[dtype]).element_size()
        assert frame_untouched(raw, rows, cols, pad, 1)
        if residual:
            assert torch.equal(h.cpu(), torch.from_numpy(want_h).to(TYPES[dtype]))
            assert frame_untouched(raw_h, rows, cols, pad, size)
        else:
            assert h is None


@pytest.mark.parametrize("cols", [1000, 8192, 40000])
def test_rms_norm_in_place(cols):
    rng = np.random.default_rng(cols)
    x = on_gpu(values(rng, (5, cols)), torch.bfloat16)
    r = on_gpu(values(rng, (5, cols)), torch.bfloat16)
    w = torch.ones(cols, dtype=torch.bfloat16, device=DEV)
    want = hv.hv_fp8_rms_norm(x, w, 1e-6, residual=r)
    for into in ("x", "residual"):
        x2, r2 = x.clone(), r.clone()
        got = hv.hv_fp8_rms_norm(x2, w, 1e-6, residual=r2, residual_out=x2 if into == "x" else r2)
        for a, b in zip(got, want):
            assert np.array_equal(bytes_of(a), bytes_of(b))


def test_rms_norm_special_rows():
    x = torch.ones(5, 300, device=DEV)
    x[0] = 0                      # nothing but zeros: codes 0, scales 1
    x[1, 7] = float("nan")        # a NaN takes its row
    x[2, 9] = float("inf")        # an infinity: NaN in its place, the rest 0
    x[3] *= 1e-20                 # squares below the smallest number: eps decides
    w = torch.ones(300, device=DEV)
    codes, scales, _ = hv.hv_fp8_rms_norm(x, w, 1e-6)
    v = codes.float().cpu().numpy()
    assert (v[0] == 0).all() and (scales[0] == 1).all()
    assert np.isnan(v[1]).all() and (scales[1] == 1).all()
    assert np.isnan(v[2, 9]) and (np.delete(v[2], 9) == 0).all()
    assert (v[3] == 448).all() and np.allclose(scales[3].cpu().numpy(), 1e-17 / 448, rtol=1e-5)
    assert (v[4] == 448).all()


# --------------------------------------------------------------------------
# gate

@pytest.mark.parametrize("joint", [False, True])
@pytest.mark.parametrize("rows,cols", SHAPES + [(64, 28672 // 4)])
@pytest.mark.parametrize("dtype", TYPES)
def test_gated(joint, rows, cols, dtype):
    rng = np.random.default_rng([rows, cols, 3])
    if joint:
        both = on_gpu(4 * values(rng, (rows, 2 * cols)), TYPES[dtype], 1)
        g, u = both[:, :cols], both[:, cols:]
    else:
        g = on_gpu(4 * values(rng, (rows, cols)), TYPES[dtype], 3, 1)
        u = on_gpu(values(rng, (rows, cols)), TYPES[dtype])
    out, raw = framed(rows, cols, torch.float8_e4m3fn, 9)
    codes, scales = hv.hv_fp8_gated(g, u, out=out)
    y = fp8.gated(g.double().cpu().numpy(), u.double().cpu().numpy())
    got = scales.cpu().numpy()
    assert np.all(np.abs(got / fp8.group_scales(y, 1) - 1) <= Y_ERROR)
    check_codes(bytes_of(codes), y, got, 1, 2 * Y_ERROR)
    assert frame_untouched(raw, rows, cols, 9, 1)


def test_gated_special_values():
    g = torch.tensor([[float("nan"), float("inf"), -float("inf"), 1000.0, -1000.0, 0.0]], device=DEV)
    codes, scales = hv.hv_fp8_gated(g, torch.ones_like(g))
    v = codes.float().cpu().numpy()[0]
    # -inf / (1 + inf) has no value; a large gate passes, a large negative one closes
    assert np.isnan(v[:3]).all() and v[3] == 448 and v[4] == 0 and v[5] == 0
    assert scales.item() == np.float32(1000) / np.float32(448)


# --------------------------------------------------------------------------
# product

def operands(rng, m, n, k, pad=0, offset=0, near=False):
    """Codes of all magnitudes (``near``: of zero and the four highest binades) and scales over several binades."""
    def codes(rows):
        if near:
            c = rng.integers(12 << 3, 127, (rows, k)) | rng.integers(0, 2, (rows, k)) << 7
            return np.where(rng.random((rows, k)) < 0.1, 0, c).astype(np.uint8)
        c = fp8.round_to_code(np.clip(rng.standard_normal((rows, k)) * 60, -448, 448))
        return np.where(rng.random((rows, k)) < 0.02, np.uint8(0), c).astype(np.uint8)
    g = -(-k // 128)
    a, b = codes(m), codes(n)
    sa = np.exp(rng.uniform(-6, 1, (m, g))).astype(np.float32)
    sb = np.exp(rng.uniform(-6, 1, (-(-n // 128), g))).astype(np.float32)
    gpu = (codes_on_gpu(a, pad, offset), torch.from_numpy(sa).to(DEV), codes_on_gpu(b, pad, offset),
           torch.from_numpy(sb).to(DEV))
    return (a, sa, b, sb), gpu


def check_product(got, host, dtype, near=True):
    c, size = fp8.matmul(*host)
    k = host[0].shape[1]
    dropped = 0 if near or dtype == "f32" else 15 * 2.0 ** -13 * size
    allowed = dropped + (k + 8) * 2.0 ** -23 * size + HALF_ULP[dtype] * np.abs(c) + (2.0 ** -25 if dtype == "f16" else 0)
    assert got.shape == c.shape and np.isfinite(got).all()
    off = np.abs(got - c) - allowed
    assert (off <= 0).all(), (np.argwhere(off > 0)[:5], off.max())


def product(m, n, k, dtype, pad=0, offset=0, out_pad=0, seed=4):
    host, gpu = operands(np.random.default_rng([m, n, k, seed]), m, n, k, pad, offset, near=dtype != "f32")
    if dtype == "f16":  # sums within the type's range
        host = (host[0], host[1] * np.float32(2.0 ** -8), *host[2:])
        gpu = (gpu[0], gpu[1] * 2.0 ** -8, *gpu[2:])
    out, raw = framed(m, n, TYPES[dtype], out_pad)
    got = hv.hv_fp8_matmul(*gpu, TYPES[dtype], out=out)
    check_product(got.double().cpu().numpy(), host, dtype)
    assert frame_untouched(raw, m, n, out_pad, torch.empty((), dtype=TYPES[dtype]).element_size())
    assert np.array_equal(bytes_of(hv.hv_fp8_matmul(*gpu, TYPES[dtype])), bytes_of(got))  # the same bits again


@pytest.mark.parametrize("k", [1, 15, 16, 64, 127, 128, 129, 240, 256, 1000, 1024, 4093])
@pytest.mark.parametrize("m,n", [(1, 1), (1, 300), (7, 129), (16, 128), (17, 16), (33, 257), (64, 100), (65, 515),
                                 (128, 256), (200, 384)])
def test_matmul_sizes(m, n, k):
    product(m, n, k, "bf16")
    product(m, n, k, "f32", pad=16, out_pad=4)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(1, 4096, 2048), (8, 1000, 4096), (31, 640, 1920), (50, 999, 777), (96, 1024, 8192),
                                   (256, 256, 256), (257, 513, 640), (300, 1100, 1280), (511, 768, 144),
                                   (1024, 1024, 1024), (130, 130, 11008), (600, 2050, 512)])
def test_matmul_types(m, n, k, dtype):
    product(m, n, k, dtype)


@pytest.mark.parametrize("m,n,k", [(1, 100, 300), (20, 200, 1024), (70, 130, 500), (300, 300, 384), (513, 260, 1023)])
def test_matmul_strides_and_offsets(m, n, k):
    for pad, offset, out_pad in ((0, 1, 1), (1, 0, 3), (13, 7, 0), (16, 16, 8), (128, 0, 5)):
        product(m, n, k, "bf16", pad, offset, out_pad)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("pad", [0, 16, 5])
@pytest.mark.parametrize("m,n,k", [(17, 4096, 1100), (32, 40, 128), (25, 5001, 777), (32, 8192, 400), (19, 9000, 300),
                                   (31, 16384, 129)])
def test_matmul_two_fragments_of_rows(m, n, k, pad, dtype):
    assert hv.matmul_launches(m, n, k, TYPES[dtype], (k + pad) % 16 == 0)[0][0].startswith("stream 2")
    product(m, n, k, dtype, pad)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(1, 1000, 20479), (4, 515, 9001), (16, 130, 20003)])
def test_matmul_few_rows_at_odd_addresses(m, n, k, dtype):
    """Long rows that are not aligned go through tiles, a single one too."""
    assert hv.matmul_launches(m, n, k, TYPES[dtype], False)[0][0] == "128x128 unaligned"
    product(m, n, k, dtype)
    product(m, n, k, dtype, pad=2, offset=3, out_pad=1)


@pytest.mark.parametrize("m,n,k", [(2048, 8448, 256), (8448, 2048, 384), (2300, 8200, 130)])
def test_matmul_larger_than_the_chip(m, n, k):
    """A round of the largest tiles, then the rest by smaller ones: the last columns, the last rows, odd edges."""
    product(m, n, k, "bf16", pad=-k % 16)


@pytest.mark.parametrize("m,n,k", [(40, 300, 9000), (100, 130, 20000), (17, 2000, 4100)])
@pytest.mark.parametrize("pad", [0, 16, 5])
def test_matmul_columns_in_parts(m, n, k, pad):
    """Few tiles and many groups: the columns are split and the parts' sums added."""
    for dtype in TYPES:
        product(m, n, k, dtype, pad)


@pytest.mark.parametrize("call,rows,cols", [("rows", 1_100_000, 24), ("gated", 1_100_000, 24), ("blocks", (1 << 27) + 300, 1),
                                            ("norm", (1 << 24) + 3000, 8), ("norm", (1 << 20) + 5, 1100)])
def test_more_rows_than_a_launch_has_workgroups(call, rows, cols):
    """The last rows, which a workgroup makes after its first ones, as a call of their own makes them."""
    x = torch.randn(rows, cols, dtype=torch.bfloat16, device=DEV)

    def run(x):
        if call == "norm":
            return hv.hv_fp8_rms_norm(x, torch.ones(cols, dtype=x.dtype, device=DEV), 1e-5, residual=x)
        return hv.hv_fp8_gated(x, x) if call == "gated" else hv.hv_fp8_quantize(x, call)

    last = (rows - 1000) // 128 * 128  # a block's first row
    whole, first, tail = run(x), run(x[:1024]), run(x[last:])
    for w, f, t in zip(whole, first, tail):
        assert np.array_equal(bytes_of(w[:len(f)]), bytes_of(f)) and np.array_equal(bytes_of(w[-len(t):]), bytes_of(t))


def test_matmul_offsets_past_32_bits():
    """Rows that start beyond 4 GiB, of every operand and of the result."""
    rng = np.random.default_rng(16)
    rows, ld, k = 70000, 65536, 200
    host, (a, sa, b, sb) = operands(rng, rows, 130, k)
    wide = torch.empty(rows, ld, dtype=torch.uint8, device=DEV)
    at = slice(rows - 40, rows)  # the oracle looks at the last rows
    for kind in ("a", "b"):
        big = wide[:, 16:16 + k].view(torch.float8_e4m3fn)
        big.view(torch.uint8).copy_(a.view(torch.uint8))
        if kind == "a":  # many rows of A: tiles; and C's rows as far apart
            out = torch.empty(rows, 40000, dtype=torch.bfloat16, device=DEV)[:, :130]
            got = hv.hv_fp8_matmul(big, sa, b, sb, out=out)[at].double().cpu().numpy()
            check_product(got, (host[0][at], host[1][at], host[2], host[3]), "bf16", near=False)
        else:  # many rows of B: few rows of A straight from memory, then tiles
            scales = torch.ones(-(-rows // 128), 2, device=DEV)
            for m in (3, 130):
                got = hv.hv_fp8_matmul(b[:m], sb[0].expand(m, 2).contiguous(), big, scales, torch.float32)
                want = (host[2][:m], np.repeat(host[3][:1], m, 0), host[0][rows - 96:], np.ones((1, 2)))
                check_product(got[:, rows - 96:].double().cpu().numpy(), want, "f32")
    x = torch.empty(rows, ld, dtype=torch.float16, device=DEV)[:, :k]
    x.copy_(torch.randn(rows, k, device=DEV))
    for tile, t in (("rows", 1), ("blocks", 128)):
        codes, scales = hv.hv_fp8_quantize(x, tile, out=big)
        y = x[rows - 112:].double().cpu().numpy()
        want = fp8.group_scales(y, t)
        assert np.array_equal(scales.cpu().numpy()[-len(want):], want)
        check_codes(bytes_of(codes[rows - 112:]), y, want, t, Q_ERROR)


def test_matmul_of_the_most_columns():
    """2^27 columns by single fragments are more workgroups than a launch may have."""
    n, k = 1 << 27, 16
    b = torch.randint(0, 0x7f, (n, k), dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
    sb = torch.rand(n // 128, 1, device=DEV)
    a, sa = hv.hv_fp8_quantize(torch.randn(1, k, device=DEV))
    got = hv.hv_fp8_matmul(a, sa, b, sb)
    for first in (0, (1 << 26) - 512, n - 1024):
        part = hv.hv_fp8_matmul(a, sa, b[first:first + 1024], sb[first // 128:first // 128 + 8])
        assert np.array_equal(bytes_of(got[:, first:first + 1024]), bytes_of(part))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("m,n,k", [(1, 500, 1024), (40, 300, 500), (150, 256, 2048), (512, 512, 768)])
def test_matmul_codes_of_all_magnitudes(m, n, k, dtype):
    host, gpu = operands(np.random.default_rng([m, n, k]), m, n, k)
    host = (host[0], host[1] * np.float32(2.0 ** -8), *host[2:])
    got = hv.hv_fp8_matmul(gpu[0], gpu[1] * 2.0 ** -8, *gpu[2:], TYPES[dtype]).double().cpu().numpy()
    check_product(got, host, dtype, near=False)
    # as a whole far nearer than the bound: a rounding's standard deviation, and 2^-14 for what the unit drops
    c, _ = fp8.matmul(*host)
    assert np.linalg.norm(got - c) <= (HALF_ULP[dtype] / 1.5 + 2.0 ** -14) * np.linalg.norm(c)


def test_matmul_drawn_sizes():
    rng = np.random.default_rng(11)
    for _ in range(40):
        m, n, k = (int(round(np.exp(rng.uniform(0, np.log(hi))))) for hi in (600, 1500, 3000))
        dtype = rng.choice(list(TYPES))
        pad, offset = (int(rng.integers(0, 40)), int(rng.integers(0, 17))) if rng.random() < 0.5 else (0, 0)
        product(m, n, k, dtype, pad, offset, int(rng.integers(0, 6)))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,n,k", [(5, 40, 300), (100, 200, 300), (300, 300, 512), (520, 520, 1024)])
def test_matmul_nan_stays_in_its_row_and_column(m, n, k, dtype):
    (a, sa, b, sb), _ = operands(np.random.default_rng(12), m, n, k)
    sa *= np.float32(2.0 ** -10)  # within half precision
    a[m // 2, k - 1] = 0x7f
    b[n // 3, 0] = 0xff
    got = hv.hv_fp8_matmul(codes_on_gpu(a, 16), torch.from_numpy(sa).to(DEV), codes_on_gpu(b, 16),
                           torch.from_numpy(sb).to(DEV), TYPES[dtype]).float().cpu().numpy()
    assert not np.isinf(got).any()
    want = np.zeros((m, n), dtype=bool)
    want[m // 2] = True
    want[:, n // 3] = True
    assert np.array_equal(np.isnan(got), want)


@pytest.mark.parametrize("m,n,k", [(5, 40, 700), (100, 200, 1100), (520, 520, 1024)])
def test_matmul_scales_of_zero_and_nan(m, n, k):
    (a, sa, b, sb), (ga, gsa, gb, gsb) = operands(np.random.default_rng(17), m, n, k)
    gsa[1] = 0
    gsa[m - 1, -1] = float("nan")
    got = hv.hv_fp8_matmul(ga, gsa, gb, gsb).float().cpu().numpy()
    assert (got[1] == 0).all() and np.isnan(got[m - 1]).all() and np.isfinite(got[:m - 1]).all()
    gsb[0, 2] = float("nan")  # the first 128 columns
    got = hv.hv_fp8_matmul(ga, gsa, gb, gsb).float().cpu().numpy()
    assert np.isnan(got[:, :128]).all() and np.isfinite(got[:m - 1, 128:]).all()


@pytest.mark.parametrize("m,n", [(3, 50), (200, 300)])
def test_matmul_without_columns_is_zero(m, n):
    a = torch.empty(m, 0, dtype=torch.float8_e4m3fn, device=DEV)
    b = torch.empty(n, 0, dtype=torch.float8_e4m3fn, device=DEV)
    sa, sb = torch.empty(m, 0, device=DEV), torch.empty(-(-n // 128), 0, device=DEV)
    out, raw = framed(m, n, torch.float32, 2)
    assert (hv.hv_fp8_matmul(a, sa, b, sb, torch.float32, out=out) == 0).all()
    assert frame_untouched(raw, m, n, 2, 4)


def test_empty_calls_do_nothing():
    for shape in ((0, 200), (3, 0), (0, 0)):
        x = torch.empty(shape, device=DEV, dtype=torch.bfloat16)
        for tile in ("rows", "blocks"):
            codes, scales = hv.hv_fp8_quantize(x, tile)
            assert codes.shape == x.shape and scales.numel() == 0
        codes, _, h = hv.hv_fp8_rms_norm(x, torch.ones(shape[1], device=DEV, dtype=torch.bfloat16), 1e-6, residual=x)
        assert codes.shape == h.shape == x.shape
        assert hv.hv_fp8_gated(x, x)[0].shape == x.shape
    a = torch.empty(0, 128, dtype=torch.float8_e4m3fn, device=DEV)
    b = torch.empty(64, 128, dtype=torch.float8_e4m3fn, device=DEV)
    sa, sb = torch.empty(0, 1, device=DEV), torch.ones(1, 1, device=DEV)
    assert hv.hv_fp8_matmul(a, sa, b, sb).shape == (0, 64)
    assert hv.hv_fp8_matmul(b, torch.ones(64, 1, device=DEV), a, sa).shape == (64, 0)


def test_leading_dimensions():
    rng = np.random.default_rng(13)
    x = torch.from_numpy(values(rng, (2, 3, 260))).to(torch.bfloat16).to(DEV)
    codes, scales = hv.hv_fp8_quantize(x)
    flat = hv.hv_fp8_quantize(x.view(6, 260))
    assert codes.shape == (2, 3, 260) and scales.shape == (2, 3, 3)
    assert np.array_equal(bytes_of(codes).reshape(6, -1), bytes_of(flat[0])) and torch.equal(scales.view(6, 3), flat[1])
    b, sb = hv.hv_fp8_quantize(torch.from_numpy(values(rng, (70, 260))).to(torch.bfloat16).to(DEV), "blocks")
    got = hv.hv_fp8_matmul(codes, scales, b, sb)
    assert got.shape == (2, 3, 70) and torch.equal(got.view(6, 70), hv.hv_fp8_matmul(*flat, b, sb))
    one = hv.hv_fp8_matmul(codes[0, 0], scales[0, 0], b, sb)
    assert one.shape == (70,) and np.allclose(one.float().cpu(), got[0, 0].float().cpu(), rtol=2 ** -7, atol=1e-3)


# --------------------------------------------------------------------------
# streams, graphs, refusals

def test_layer_in_a_graph_on_its_own_stream():
    """norm, product, gate, product: captured once, replayed on changing inputs beside other work."""
    rng = np.random.default_rng(14)
    d, f, m = 512, 768, 24
    w1 = hv.hv_fp8_quantize(torch.from_numpy(values(rng, (2 * f, d))).to(torch.bfloat16).to(DEV), "blocks")
    w2 = hv.hv_fp8_quantize(torch.from_numpy(values(rng, (d, f))).to(torch.bfloat16).to(DEV), "blocks")
    norm = torch.ones(d, dtype=torch.bfloat16, device=DEV)
    ws = hv.Workspace(DEV)
    ws.get(1 << 22)
    x, r = (torch.zeros(m, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))

    def layer():
        codes, scales, h = hv.hv_fp8_rms_norm(x, norm, 1e-6, residual=r)
        both = hv.hv_fp8_matmul(codes, scales, *w1, workspace=ws)
        codes, scales = hv.hv_fp8_gated(both[:, :f], both[:, f:])
        return hv.hv_fp8_matmul(codes, scales, *w2, torch.float32, workspace=ws), h

    side = torch.cuda.Stream(DEV)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = layer()
        for trip in range(4):
            x.copy_(torch.from_numpy(values(rng, (m, d))).to(torch.bfloat16))
            r.copy_(torch.from_numpy(values(rng, (m, d))).to(torch.bfloat16))
            graph.replay()
            kept = [t.clone() for t in got]
            want = layer()
            side.synchronize()
            for a, b in zip(kept, want):
                assert torch.equal(a, b), trip


def test_binding_refusals():
    x = torch.ones(4, 256, device=DEV, dtype=torch.bfloat16)
    w = torch.ones(256, device=DEV, dtype=torch.bfloat16)
    q, s = hv.hv_fp8_quantize(x)
    b, sb = hv.hv_fp8_quantize(torch.ones(130, 256, device=DEV, dtype=torch.bfloat16), "blocks")
    calls = [
        (lambda: hv.hv_fp8_quantize(x.cpu()), "device tensor"),
        (lambda: hv.hv_fp8_quantize(x.double()), "expected one of"),
        (lambda: hv.hv_fp8_quantize(x.t()), "adjacent"),
        (lambda: hv.hv_fp8_quantize(x[:1].expand(4, 256)), "overlap"),
        (lambda: hv.hv_fp8_quantize(x, "columns"), "unknown tile"),
        (lambda: hv.hv_fp8_quantize(x.view(2, 2, 256), "blocks"), "two-dimensional"),
        (lambda: hv.hv_fp8_quantize(x, out=q[:3]), "shape"),
        (lambda: hv.hv_fp8_quantize(x, scales=s[:, :1]), "shape"),
        (lambda: hv.hv_fp8_rms_norm(x, w[:255], 1e-6), "shape"),
        (lambda: hv.hv_fp8_rms_norm(x, w.float(), 1e-6), "expected one of"),
        (lambda: hv.hv_fp8_rms_norm(x, w, 1e-6, residual=x[:2]), "shape"),
        (lambda: hv.hv_fp8_rms_norm(x, w, 1e-6, residual_out=x), "without a residual"),
        (lambda: hv.hv_fp8_gated(x, x[:, :128]), "shape"),
        (lambda: hv.hv_fp8_gated(x, x.float()), "expected one of"),
        (lambda: hv.hv_fp8_matmul(q, s, b[:, :255], sb), "needs"),
        (lambda: hv.hv_fp8_matmul(q, s[:3], b, sb), "a_scales has shape"),
        (lambda: hv.hv_fp8_matmul(q, s, b, sb[:1]), "b_scales has shape"),
        (lambda: hv.hv_fp8_matmul(q, s.double(), b, sb), "expected one of"),
        (lambda: hv.hv_fp8_matmul(q, torch.ones(4, 4, device=DEV)[:, ::2], b, sb), "adjacent"),
        (lambda: hv.hv_fp8_matmul(q, torch.ones(4, 4, device=DEV)[:, :2], b, sb), "contiguous"),
        (lambda: hv.hv_fp8_matmul(x, s, b, sb), "expected one of"),
        (lambda: hv.hv_fp8_matmul(q, s, b, sb, torch.float64), "expected one of"),
        (lambda: hv.hv_fp8_matmul(q, s, b, sb, out=torch.empty(4, 129, device=DEV, dtype=torch.bfloat16)), "shape"),
    ]
    for call, words in calls:
        with pytest.raises(ValueError, match=words):
            call()
    with pytest.raises(hv.HVError, match="eps"):
        hv.hv_fp8_rms_norm(x, w, float("nan"))
    assert hv.hv_fp8_matmul(q, s, b, sb).shape == (4, 130)
