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
    for m, n, k in ((0, 100, 100), (100, 0, 100), (1 << 31, 8, 8), (8, 8, (1 << 24) + 1)):
        assert hv.lib.hv_fp8_matmul_workspace_bytes(m, n, k) == 0
    for m in (1, 2, 16, 17, 64, 65, 128, 300, 2048, 100000):
        for n, k in ((1, 1), (128, 28672), (1000, 1000), (8192, 8192), (57344, 128)):
            need = hv.lib.hv_fp8_matmul_workspace_bytes(m, n, k)
            assert need % 256 == 0
            if need:
                args = {**MATMUL, "m": m, "n": n, "k": k, "ld_a": k, "ld_b": k, "ld_c": n}
                for change in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=P + 8)):
                    assert hv.lib.hv_fp8_matmul(*{**args, **change}.values(), None) == hv.HV_ERR_WORKSPACE
