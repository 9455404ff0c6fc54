"""What the binding of the cache, the attention and the adapters does around the library's calls.  None of it needs a
GPU: tensors in host memory say that they are on one, and a recorder stands in for the library."""
import pytest
import torch
from torch.autograd import forward_ad

import test_fp8_binding as base
from paper_2510_23938_amd import hv  # noqa: E402  (a missing library fails the run, never skips it)

E4M3, F32, I32 = torch.float8_e4m3fn, torch.float32, torch.int32
LIBRARY = {"write": "hv_fp8_cache_write", "attention": "hv_fp8_attention", "adapters": "hv_fp8_adapters"}


def tensor(*shape, dtype=torch.bfloat16):
    """16-byte aligned, as the GPU's allocations are."""
    raw = torch.zeros(int(torch.Size(shape).numel()) * torch.empty((), dtype=dtype).element_size() + 16, dtype=torch.uint8)
    raw = raw[-raw.data_ptr() % 16:][:raw.numel() - 16]
    return raw.view(dtype).view(shape).as_subclass(base.OnGpu1)


def parts():
    return [tensor(4, 2, 32, 64, dtype=E4M3), tensor(4, 2, 2, dtype=F32), tensor(4, 2, 2, 64, 16, dtype=E4M3),
            tensor(4, 2, 2, dtype=F32)]


def arguments():
    cache = hv.Fp8Cache(*parts())
    batch = dict(starts=tensor(4, dtype=I32), lengths=tensor(3, dtype=I32), pages=tensor(3, 5, dtype=I32))
    return {"write": (hv.hv_fp8_cache_write, dict(cache=cache, k=tensor(6, 2, 64), v=tensor(6, 2, 64), **batch)),
            "attention": (hv.hv_fp8_attention, dict(q=tensor(6, 4, 64), cache=cache, **batch, out=tensor(6, 4, 64))),
            "adapters": (hv.hv_fp8_adapters, dict(y=tensor(6, 128), x=tensor(6, 256, dtype=E4M3),
                                                  x_scales=tensor(6, 2, dtype=F32), down=tensor(3, 16, 256),
                                                  up=tensor(3, 128, 16), index=tensor(6, dtype=I32),
                                                  factors=tensor(3, dtype=F32), out=tensor(6, 128)))}


class Library(base.Library):
    need = 0

    def hv_fp8_attention_workspace_bytes(self, *args):
        return self.need

    hv_fp8_adapters_workspace_bytes = hv_fp8_attention_workspace_bytes


@pytest.mark.parametrize("operator", LIBRARY)
@pytest.mark.parametrize("current", [0, 1])
def test_the_tensors_gpu_is_current_for_the_call(monkeypatch, operator, current):
    library = Library(monkeypatch, current)
    call, args = arguments()[operator]
    call(**args)
    assert library.calls == [(LIBRARY[operator], 1, 1001)]
    assert library.current == current


@pytest.mark.parametrize("operator", ["attention", "adapters"])
@pytest.mark.parametrize("device", ["cpu", "cuda:0"])
def test_scratch_elsewhere_is_refused(monkeypatch, operator, device):
    library = Library(monkeypatch, 1)
    library.need = 4096
    monkeypatch.setattr(hv.Workspace, "get", lambda self, nbytes: torch.empty(nbytes, dtype=torch.uint8))
    call, args = arguments()[operator]
    with pytest.raises(ValueError, match="workspace"):
        call(**args, workspace=hv.Workspace(device))
    assert library.calls == []


@pytest.mark.parametrize("operator", LIBRARY)
def test_gradients_are_refused_where_they_would_be_lost(monkeypatch, operator):
    library = Library(monkeypatch, 1)
    wide = [k for k, v in arguments()[operator][1].items()
            if isinstance(v, torch.Tensor) and v.dtype in (torch.bfloat16, torch.float32)]
    assert wide
    for name in wide:
        call, args = arguments()[operator]
        args[name].requires_grad_()
        with pytest.raises(ValueError, match=f"{name} requires a gradient"):
            call(**args)
        assert library.calls == []
        with torch.no_grad():
            call(**args)
        assert len(library.calls) == 1
        library.calls.clear()


@pytest.mark.parametrize("operator", LIBRARY)
def test_forward_mode_tangents_are_refused(monkeypatch, operator):
    library = Library(monkeypatch, 1)
    call, args = arguments()[operator]
    wide = [k for k, v in args.items() if isinstance(v, torch.Tensor) and v.dtype in (torch.bfloat16, F32)]
    assert wide
    with forward_ad.dual_level():
        call(**args)
        assert len(library.calls) == 1
        for name in wide:
            args = arguments()[operator][1]
            args[name] = forward_ad.make_dual(args[name], torch.ones_like(args[name])).as_subclass(base.OnGpu1)
            with pytest.raises(ValueError, match=f"{name} carries a tangent"), torch.no_grad():
                call(**args)
    assert len(library.calls) == 1


REFUSED = [
    ("write", "k", lambda t: tensor(6, 3, 64), "k has shape"), ("write", "k", lambda t: tensor(6, 2, 48), "k has shape"),
    ("write", "v", lambda t: tensor(5, 2, 64), "v has shape"), ("write", "v", lambda t: tensor(6, 2, 64, dtype=F32), "v is"),
    ("write", "k", lambda t: tensor(6, 2, 128)[:, :, ::2], "adjacent"), ("write", "k", lambda t: tensor(6, 128), "k has shape"),
    ("write", "k", lambda t: tensor(6, 2, 64, dtype=torch.float64), "k is"),
    ("attention", "q", lambda t: tensor(6, 3, 64), "q has shape"), ("attention", "q", lambda t: tensor(6, 4, 80), "q has shape"),
    ("attention", "q", lambda t: tensor(6, 0, 64), "q has shape"),
    ("attention", "q", lambda t: tensor(6, 4, 64, dtype=F32), "q is"),
    ("attention", "out", lambda t: tensor(6, 4, 64, dtype=torch.float16), "out is"),
    ("attention", "out", lambda t: tensor(5, 4, 64), "out has shape"),
    *((op, "starts", lambda t: tensor(3, dtype=I32), "starts") for op in ("write", "attention")),
    *((op, "starts", lambda t: tensor(4, dtype=torch.int64), "starts is") for op in ("write", "attention")),
    *((op, "lengths", lambda t: tensor(6, dtype=I32)[::2], "contiguous") for op in ("write", "attention")),
    *((op, "pages", lambda t: tensor(2, 5, dtype=I32), "pages has shape") for op in ("write", "attention")),
    *((op, "pages", lambda t: tensor(5, 3, dtype=I32).t(), "adjacent") for op in ("write", "attention")),
    *((op, "pages", lambda t: torch.zeros(3, 5, dtype=I32), "pages") for op in ("write", "attention")),
    ("adapters", "x", lambda t: tensor(5, 256, dtype=E4M3), "x has shape"), ("adapters", "x", lambda t: tensor(6, 256), "x is"),
    ("adapters", "x_scales", lambda t: tensor(6, 3, dtype=F32), "x_scales"),
    ("adapters", "down", lambda t: tensor(3, 16, 200), "down"), ("adapters", "up", lambda t: tensor(3, 128, 8), "up"),
    ("adapters", "up", lambda t: tensor(3, 128, 16, dtype=torch.float16), "one type"),
    ("adapters", "down", lambda t: tensor(3, 16, 256, dtype=F32), "down is"),
    ("adapters", "down", lambda t: tensor(3, 256, 16).transpose(1, 2), "contiguous"),
    ("adapters", "index", lambda t: tensor(5, dtype=I32), "index"),
    ("adapters", "index", lambda t: tensor(6, dtype=torch.int64), "index is"),
    ("adapters", "factors", lambda t: tensor(2, dtype=F32), "factors"),
    ("adapters", "out", lambda t: tensor(6, 127), "out has shape"),
]


@pytest.mark.parametrize("operator,name,change,words", REFUSED, ids=lambda v: v if isinstance(v, str) else "")
def test_refused(monkeypatch, operator, name, change, words):
    library = Library(monkeypatch, 1)
    call, args = arguments()[operator]
    args[name] = change(args[name])
    with pytest.raises(ValueError, match=words):
        call(**args)
    assert library.calls == []


@pytest.mark.parametrize("window,sinks", [(-1, 0), (1 << 32, 0), (5, -1), (5, 1 << 32)])
def test_windows_refused(monkeypatch, window, sinks):
    library = Library(monkeypatch, 1)
    call, args = arguments()["attention"]
    with pytest.raises(ValueError, match="window"):
        call(**args, window=window, sinks=sinks)
    assert library.calls == []


def test_caches_refused():
    def bad(i, t):
        p = parts()
        p[i] = t
        return p

    for words, p in (("k_codes has shape", bad(0, tensor(4, 2, 64, dtype=E4M3))),
                     ("v_codes has shape", bad(2, tensor(4, 2, 2, 16, 64, dtype=E4M3))),
                     ("k_codes is", bad(0, tensor(4, 2, 32, 64, dtype=torch.uint8))),
                     ("k_scales must", bad(1, tensor(4, 2, 3, dtype=F32))), ("v_scales is", bad(3, tensor(4, 2, 2))),
                     ("contiguous", bad(0, tensor(4, 2, 64, 32, dtype=E4M3).transpose(2, 3))),
                     ("16-byte", bad(0, tensor(4 * 2 * 2056 + 8, dtype=E4M3).as_strided((4, 2, 32, 64), (4112, 2056, 64, 1)))),
                     ("16-byte", bad(2, tensor(4 * 4096 + 8, dtype=E4M3)[8:].view(4, 2, 2, 64, 16))),
                     ("16-byte|shape", bad(0, torch.zeros(4, 2, 32, 64).to(E4M3)))):
        with pytest.raises(ValueError, match=words if "shape" not in words or "has" in words else "device"):
            hv.Fp8Cache(*p)
    for shape in ((4, 2, 0, 64), (4, 0, 32, 64), (4, 2, 24, 64), (4, 2, 32, 8), (4, 2, 32, 272), (4, 2, 65552, 16)):
        pages, heads, tokens, dim = shape
        with pytest.raises(ValueError, match="a cache of"):
            hv.Fp8Cache(tensor(*shape, dtype=E4M3), tensor(pages, heads, tokens // 16, dtype=F32),
                        tensor(pages, heads, tokens // 16, dim, 16, dtype=E4M3),
                        tensor(pages, heads, tokens // 16, dtype=F32))
    with pytest.raises(ValueError, match="page_tokens"):
        hv.Fp8Cache.empty(4, 2, 40, 64, device="cpu")


@pytest.mark.parametrize("name", ["k_codes", "k_scales", "v_codes", "v_scales", "pages", "kv_heads", "page_tokens", "head_dim", "device"])
def test_a_caches_parts_stay(name):
    """Calls go to the addresses and sizes that the cache was made with: another tensor in one's place would be neither
    checked nor used, and the one before it freed under them."""
    cache = hv.Fp8Cache(*parts())
    was = getattr(cache, name)
    with pytest.raises(AttributeError, match="another Fp8Cache"):
        setattr(cache, name, was)
    with pytest.raises(AttributeError, match="another Fp8Cache"):
        delattr(cache, name)
    assert getattr(cache, name) is was


def test_strides_as_the_library_takes_them(monkeypatch):
    """Keys and values of one product's rows, a table's rows apart, pages of a pool that holds both."""
    seen = {}

    class Recorder(Library):
        def __getattr__(self, name):
            def call(*args):
                seen[name] = args
                return hv.HV_OK
            return call

    Recorder(monkeypatch, 1)
    both = tensor(4, 2, 2, 32, 64, dtype=E4M3)
    p = parts()
    cache = hv.Fp8Cache(both[:, 0], p[1], p[2], p[3])
    assert (cache._struct.k_page, cache._struct.k_head, cache._struct.v_page, cache._struct.v_head) == (8192, 2048, 4096, 2048)
    rows = tensor(6, 512)
    k, v = rows[:, 256:384].view(6, 2, 64), rows[:, 384:].view(6, 2, 64)
    table = tensor(3, 9, dtype=I32)[:, :5]
    hv.hv_fp8_cache_write(cache, k, v, tensor(4, dtype=I32), tensor(3, dtype=I32), table)
    _, batch, _, k_ptr, k_token, k_head, v_ptr, v_token, v_head, tokens, _ = seen["hv_fp8_cache_write"]
    assert (k_ptr - rows.data_ptr(), k_token, k_head, v_ptr - k_ptr, v_token, v_head, tokens) == (512, 512, 64, 256, 512, 64, 6)
    assert (batch._obj.count, batch._obj.columns, batch._obj.ld_pages) == (3, 5, 9)
    one = hv.hv_fp8_attention(rows[:1, :256].view(1, 4, 64), cache, tensor(2, dtype=I32), tensor(1, dtype=I32),
                              tensor(1, 5, dtype=I32), out=tensor(1, 4, 64))
    assert one.shape == (1, 4, 64) and seen["hv_fp8_attention"][4:8] == (256, 64, 1, 4)
