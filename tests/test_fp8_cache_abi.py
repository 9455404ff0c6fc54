"""Argument checks of the 8-bit cache's, attention's and adapters' C ABI: each fails before any HIP call, so none needs
a GPU."""
import ctypes

import pytest

from paper_2510_23938_amd import hv  # noqa: E402  (a missing library fails the run, never skips it)

P, Q = 0x10000, 0x20000
CACHE = dict(k_codes=P, k_scales=P, v_codes=P, v_scales=P, pages=4, kv_heads=2, page_tokens=32, head_dim=64,
             k_page=4096, k_head=2048, v_page=4096, v_head=2048)
BATCH = dict(starts=P, lengths=P, pages=P, count=2, columns=3, ld_pages=3)
WRITE = dict(type=hv.HV_BF16, k=P, k_token=128, k_head=64, v=P, v_token=128, v_head=64, tokens=5)
ATTENTION = dict(type=hv.HV_BF16, q=P, q_token=256, q_head=64, tokens=5, heads=4, scale=0.125, window=0, sinks=0, out=Q,
                 out_token=256, out_head=64, workspace=P, workspace_bytes=1 << 40)
ADAPTERS = dict(type=hv.HV_BF16, adapter_type=hv.HV_BF16, y=P, ld_y=256, x=P, ld_x=512, x_scales=P, down=P, up=P,
                factors=P, index=P, adapters=3, rank=16, m=4, n=256, k=512, out=Q, ld_out=256, workspace=P,
                workspace_bytes=1 << 40)


def call(name, change):
    def args(good):
        return {k: change.get(k, v) for k, v in good.items()}

    if name == "adapters":
        return hv.lib.hv_fp8_adapters(*args(ADAPTERS).values(), None)
    cache = hv.hv_fp8_cache(**{k: change.get("cache_" + k, v) for k, v in CACHE.items()})
    batch = hv.hv_fp8_batch(**{k: change.get("batch_" + k, v) for k, v in BATCH.items()})
    f, good = {"write": (hv.lib.hv_fp8_cache_write, WRITE), "attention": (hv.lib.hv_fp8_attention, ATTENTION)}[name]
    c = None if change.get("no_cache") else ctypes.byref(cache)
    b = None if change.get("no_batch") else ctypes.byref(batch)
    return f(c, b, *args(good).values(), None)


BOTH = ("write", "attention")
BAD = [
    ("write", dict(type=3), b"element type"), ("write", dict(type=-1), b"element type"),
    ("attention", dict(type=hv.HV_F32), b"neither"), ("adapters", dict(type=3), b"element type"),
    ("adapters", dict(adapter_type=hv.HV_F32), b"neither"),
    *((n, {"no_cache": True}, b"cache is NULL") for n in BOTH), *((n, {"no_batch": True}, b"batch is NULL") for n in BOTH),
    *((n, {"cache_" + p: None}, b"is NULL") for n in BOTH for p in ("k_codes", "k_scales", "v_codes", "v_scales")),
    *((n, {"cache_" + p: P + 8}, b"16-byte") for n in BOTH for p in ("k_codes", "v_codes")),
    *((n, {"cache_k_scales": P + 2}, b"aligned") for n in BOTH),
    *((n, {"batch_" + p: None}, b"is NULL") for n in BOTH for p in ("starts", "lengths", "pages")),
    *((n, {"batch_" + p: P + 2}, b"aligned") for n in BOTH for p in ("starts", "lengths", "pages")),
    *((n, {"cache_head_dim": d}, b"head_dim") for n in BOTH for d in (0, 8, 24, 272)),
    *((n, {"cache_page_tokens": t}, b"page_tokens") for n in BOTH for t in (0, 8, 40, 65552)),
    *((n, {"cache_kv_heads": h}, b"kv_heads") for n in BOTH for h in (0, 65536)),
    *((n, {"cache_pages": 1 << 31}, b"pages") for n in BOTH),
    *((n, {"cache_" + p: 2040}, b"16 bytes apart") for n in BOTH for p in ("k_page", "k_head", "v_page", "v_head")),
    *((n, {"cache_" + p: 2032}, b"overlap") for n in BOTH for p in ("k_page", "k_head", "v_page", "v_head")),
    *((n, {"cache_" + p: 1 << 41}, b"limit") for n in BOTH for p in ("k_page", "v_head")),
    *((n, {"batch_count": 65537}, b"sequences") for n in BOTH),
    *((n, {"batch_columns": (1 << 25) + 1, "batch_ld_pages": 1 << 26}, b"columns") for n in BOTH),
    *((n, {"batch_ld_pages": 2}, b"ld_pages") for n in BOTH),
    *(("write", {p: None}, b"is NULL") for p in "kv"), *(("write", {p: P + 1}, b"aligned") for p in "kv"),
    *(("write", {p: 63}, b"overlap") for p in ("k_token", "k_head", "v_token", "v_head")),
    ("write", dict(tokens=(1 << 29) + 1), b"tokens"), ("write", dict(k_token=1 << 41), b"limit"),
    *(("attention", {p: None}, b"is NULL") for p in ("q", "out")),
    *(("attention", {p: P + 1}, b"aligned") for p in ("q", "out")),
    *(("attention", {p: 63}, b"overlap") for p in ("q_token", "q_head", "out_token", "out_head")),
    *(("attention", {"heads": h}, b"heads") for h in (0, 3, 1 << 31)),
    ("attention", dict(tokens=(1 << 28) + 1), b"tokens"),
    *(("attention", {"scale": s}, b"scale") for s in (0.0, -1.0, float("nan"), float("inf"), 3e38, 1e-39)),
    *(("adapters", {p: None}, b"is NULL") for p in ("y", "x", "x_scales", "down", "up", "index", "out")),
    *(("adapters", {p: P + 1}, b"aligned") for p in ("y", "x_scales", "down", "up", "factors", "index", "out")),
    *(("adapters", {p: 255}, b"below its") for p in ("ld_y", "ld_out")), ("adapters", dict(ld_x=511), b"below its"),
    *(("adapters", {"rank": r}, b"rank") for r in (0, 1025)), ("adapters", dict(adapters=1 << 31), b"adapters"),
    *(("adapters", {p: (1 << 27) + 1}, b"limit") for p in ("m", "n")),
    ("adapters", dict(k=(1 << 24) + 1), b"limit"),
    ("adapters", dict(m=1 << 20, n=(1 << 20) + 1, ld_y=1 << 21, ld_out=1 << 21), b"2^40"),
    ("adapters", dict(out=P, ld_out=300), b"overlaps"),
]


@pytest.mark.parametrize("name,change,words", BAD, ids=lambda v: str(v)[:40])
def test_refused_before_launch(name, change, words):
    assert call(name, change) == hv.HV_ERR_INVALID_ARG
    assert words in hv.lib.hv_last_error(), hv.lib.hv_last_error()


def test_calls_with_nothing_to_write_need_no_pointers():
    none = dict.fromkeys(("k", "v", "q", "out", "y", "x", "x_scales", "down", "up", "factors", "index", "workspace"))
    for name in BOTH:
        assert call(name, {**none, "tokens": 0}) == hv.HV_OK
        assert call(name, {**none, "batch_count": 0, "batch_starts": None, "batch_lengths": None}) == hv.HV_OK
    assert call("write", {**none, "cache_pages": 0, "cache_k_codes": None}) == hv.HV_OK
    assert call("write", {**none, "batch_columns": 0, "batch_pages": None}) == hv.HV_OK
    for p in ("m", "n"):
        assert call("adapters", {**none, "k": 512, p: 0}) == hv.HV_OK


def test_places_nested_either_way():
    """Pages within heads and heads within pages pass the checks (and the call ends at what is checked after them)."""
    for k_page, k_head in ((4096, 2048), (2048, 8192), (6144, 2048), (2048, 8208)):
        assert call("write", dict(cache_k_page=k_page, cache_k_head=k_head, k=None)) == hv.HV_ERR_INVALID_ARG
        assert hv.lib.hv_last_error() == b"k is NULL"
    for token, head in ((128, 64), (64, 320), (200, 70)):
        assert call("write", dict(k_token=token, k_head=head, v=None)) == hv.HV_ERR_INVALID_ARG
        assert hv.lib.hv_last_error() == b"v is NULL"


def test_attention_workspace():
    size = hv.lib.hv_fp8_attention_workspace_bytes
    for bad in ((0, 100, 5, 4, 2, 64), (2, 0, 5, 4, 2, 64), (2, 100, 0, 4, 2, 64), (2, 100, 5, 3, 2, 64),
                (2, 100, 5, 4, 2, 65), (65537, 100, 5, 4, 2, 64), (2, 1 << 31, 5, 4, 2, 64), (2, 100, 1 << 30, 4, 2, 64)):
        assert size(*bad, 0, 0) == 0
    assert size(1, 1536, 1, 8, 1, 128, 0, 0) == 0 and size(1, 1 << 20, 1, 8, 1, 128, 512, 4) == 0
    for sequences, tokens, heads in ((1, 1, 4), (3, 40, 8), (64, 64, 16), (1, 3000, 2)):
        need = size(sequences, 1 << 20, tokens, heads, 2, 64, 0, 0)
        assert need > 0 and need % 256 == 0
        args = {"batch_count": sequences, "batch_columns": 1 << 15, "batch_ld_pages": 1 << 15, "tokens": tokens,
                "heads": heads, "q_token": heads * 64, "out_token": heads * 64}
        for change in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=P + 8)):
            assert call("attention", {**args, **change}) == hv.HV_ERR_WORKSPACE


def test_adapters_workspace():
    size = hv.lib.hv_fp8_adapters_workspace_bytes
    for bad in ((3, 0, 4, 512), (3, 16, 0, 512), (0, 16, 4, 512), (3, 16, 4, 0), (3, 2000, 4, 512), (1 << 31, 16, 4, 512)):
        assert size(*bad) == 0
    for adapters, rank, m, k in ((1, 1, 1, 1), (3, 16, 4, 512), (40, 64, 40, 8192), (8, 16, 2048, 8192), (2, 1024, 9, 4093)):
        need = size(adapters, rank, m, k)
        assert need > 0 and need % 256 == 0 and need >= 4 * m * rank
        args = dict(adapters=adapters, rank=rank, m=m, k=k, ld_x=k)
        for change in (dict(workspace=None), dict(workspace_bytes=need - 1), dict(workspace=P + 8)):
            assert call("adapters", {**args, **change}) == hv.HV_ERR_WORKSPACE
