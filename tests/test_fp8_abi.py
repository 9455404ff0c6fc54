"""Argument checks of the 8-bit operators' C ABI: each fails before any HIP call, so none needs a GPU."""
import pytest

from paper_2510_23938_amd import hv  # noqa: E402  (a missing library fails the run, never skips it)

P, Q = 0x10000, 0x20000
QUANTIZE = dict(type=hv.HV_BF16, x=P, ld_x=256, rows=4, cols=256, tile=1, codes=Q, ld_codes=256, scales=P)
NORM = dict(type=hv.HV_BF16, x=P, ld_x=256, residual=P, ld_residual=256, weight=P, eps=1e-6, rows=4, cols=256,
            residual_out=Q, ld_out=256, codes=Q, ld_codes=256, scales=P)
GATED = dict(type=hv.HV_BF16, gate=P, ld_gate=256, up=P, ld_up=256, rows=4, cols=256, codes=Q, ld_codes=256, scales=P)
MATMUL = dict(type=hv.HV_BF16, a=P, ld_a=256, a_scales=P, b=P, ld_b=256, b_scales=P, m=4, n=256, k=256, c=Q, ld_c=256,
              workspace=P, workspace_bytes=1 << 40)
CALLS = {"quantize": (hv.lib.hv_fp8_quantize, QUANTIZE), "norm": (hv.lib.hv_fp8_rms_norm, NORM),
         "gated": (hv.lib.hv_fp8_gated, GATED), "matmul": (hv.lib.hv_fp8_matmul, MATMUL)}

BAD = [
    *((c, dict(type=t), b"element type") for c in CALLS for t in (-1, 3)),
    *((c, {p: None}, b"is NULL") for c, ps in (("quantize", ("x", "codes", "scales")),
                                               ("norm", ("x", "weight", "codes", "scales")),
                                               ("gated", ("gate", "up", "codes", "scales")),
                                               ("matmul", ("a", "b", "a_scales", "b_scales", "c"))) for p in ps),
    *((c, {p: P + 1}, b"aligned") for c, ps in (("quantize", ("x", "scales")), ("norm", ("x", "residual", "weight")),
                                                ("gated", ("gate", "up")), ("matmul", ("a_scales", "c"))) for p in ps),
    *((c, {p: 255}, b"below its") for c, ps in (("quantize", ("ld_x", "ld_codes")),
                                                ("norm", ("ld_x", "ld_residual", "ld_out", "ld_codes")),
                                                ("gated", ("ld_gate", "ld_up")), ("matmul", ("ld_a", "ld_b", "ld_c")))
      for p in ps),
    *((c, {p: (1 << 31) + 1}, b"limit") for c, ps in (("quantize", ("ld_x", "rows", "cols")), ("norm", ("rows", "cols")),
                                                      ("gated", ("rows", "ld_up")), ("matmul", ("m", "n", "k", "ld_c")))
      for p in ps),
    ("quantize", dict(tile=0), b"tile_rows"), ("quantize", dict(tile=64), b"tile_rows"),
    ("norm", dict(eps=-1.0), b"eps"), ("norm", dict(eps=float("nan")), b"eps"),
    ("norm", dict(residual=None), b"together"), ("norm", dict(residual_out=None), b"together"),
    ("norm", dict(residual_out=P, ld_out=300), b"overlaps"),
]


@pytest.mark.parametrize("call,change,words", BAD)
def test_refused_before_launch(call, change, words):
    f, good = CALLS[call]
    assert f(*{**good, **change}.values(), None) == hv.HV_ERR_INVALID_ARG
    assert words in hv.lib.hv_last_error()


def test_empty_calls_need_no_pointers():
    for rows, cols in ((0, 256), (4, 0), (0, 0)):
        assert hv.lib.hv_fp8_quantize(hv.HV_F32, None, 0, rows, cols, 128, None, 0, None, None) == hv.HV_OK
        assert hv.lib.hv_fp8_gated(hv.HV_F16, None, 0, None, 0, rows, cols, None, 0, None, None) == hv.HV_OK
        assert hv.lib.hv_fp8_rms_norm(hv.HV_BF16, None, 0, None, 0, None, 0.0, rows, cols, None, 0, None, 0, None,
                                      None) == hv.HV_OK
    for m, n in ((0, 5), (5, 0)):
        assert hv.lib.hv_fp8_matmul(hv.HV_BF16, None, 0, None, None, 0, None, m, n, 128, None, 0, None, 0,
                                    None) == hv.HV_OK


def test_workspace_sizes():
    size = hv.lib.hv_fp8_matmul_workspace_bytes
    for m, n, k in ((0, 100, 100), (100, 0, 100), (1 << 31, 8, 8), (8, 8, (1 << 24) + 1)):
        assert size(hv.HV_BF16, 1, m, n, k) == 0
    assert size(7, 1, 100, 100, 1 << 20) == 0 and size(hv.HV_BF16, 1, 100, 100, 1 << 20) > 0
    for t in (hv.HV_BF16, hv.HV_F32):
        for m in (1, 2, 16, 17, 64, 65, 128, 300, 2048, 100000):
            for n, k in ((1, 1), (128, 28672), (1000, 1000), (8192, 8192), (57344, 128), (500, 8191)):
                for aligned in (0, 1):
                    need = size(t, aligned, m, n, k)
                    assert need % 256 == 0
                    if need:
                        ld = k + -k % 16 + (0 if aligned else 1)
                        args = {**MATMUL, "type": t, "m": m, "n": n, "k": k, "ld_a": ld, "ld_b": ld, "ld_c": n}
                        for change in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=P + 8)):
                            assert hv.lib.hv_fp8_matmul(*{**args, **change}.values(), None) == hv.HV_ERR_WORKSPACE


def test_which_kernels_a_product_takes():
    """The rule's cases: each kernel is taken for some size, and each part covers its rows and columns."""
    bf16, f32 = hv.torch.bfloat16, hv.torch.float32
    taken = {}
    for dtype in (bf16, f32):
        for aligned in (True, False):
            for m in (1, 4, 8, 16, 17, 32, 33, 64, 150, 256, 333, 1000, 2048, 4096):
                for n in (64, 1024, 4096, 5001, 11008, 16384, 28672):
                    for k in (0, 100, 1024, 4093, 28672):
                        parts = hv.matmul_launches(m, n, k, dtype, aligned)
                        packed = parts[0][0] == "pack"
                        if packed:
                            assert not aligned and parts[0][1:] == (m, n, 1)
                            taken["pack"] = {False}
                            parts = parts[1:]
                        assert sum(r * c for _, r, c, _ in parts) == m * n
                        if len(parts) == 2:
                            (_, r0, c0, _), (_, r1, c1, _) = parts
                            assert (r0 == r1 == m and c0 + c1 == n and c0 % 256 == 0) or \
                                (c0 == c1 == n and r0 + r1 == m and r0 % 256 == 0)
                        for kind, _, _, splits in parts:
                            taken.setdefault(kind, set()).add(splits > 1)
                            assert splits == 1 or kind.startswith("128x128")
                            stream = kind.startswith("stream")
                            assert stream if m <= 16 and k > 0 and aligned else not stream or m <= 32
                            assert kind.startswith("stream 2") == (stream and m > 16)
                            assert (kind == "128x128 unaligned") == (not aligned and not packed and not stream and k > 0)
    assert set(taken) == set(hv._MATMUL_KINDS)
    assert taken["128x128"] == taken["128x128 unaligned"] == {True, False}
    assert [p[0] for p in hv.matmul_launches(2048, 28672, 8192)] == ["256x256", "256x128"]
    assert hv.matmul_launches(0, 5, 5) == []
    assert hv.lib.hv_fp8_matmul_launches(0, 1, 1, 1, 1, None, None, None, None, None) == hv.HV_ERR_INVALID_ARG
