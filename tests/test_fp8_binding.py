"""What the binding of the 8-bit operators does around the library's calls.  None of it needs a GPU: tensors in host
memory say that they are on one, and a recorder stands in for the library."""
import contextlib
import gc
import weakref

import pytest
import torch

from paper_2510_23938_amd import hv  # noqa: E402  (a missing library fails the run, never skips it)

OPERATORS = ("quantize", "rms_norm", "gated", "matmul")


class OnGpu1(torch.Tensor):
    """A tensor in host memory that says it is on the second GPU."""
    device = property(lambda self: torch.device("cuda", 1))
    is_cuda = True
    get_device = lambda self: 1  # noqa: E731


def tensor(*shape, dtype=torch.bfloat16, fill=1.0):
    return torch.full(shape, fill, dtype=torch.float32).to(dtype).as_subclass(OnGpu1)


def arguments():
    """{operator: (function, arguments)}: small calls with every output given."""
    e4m3, f32 = torch.float8_e4m3fn, torch.float32
    x, w, s = tensor(4, 256), tensor(256), tensor(4, 2, dtype=f32)
    q, b, sb = tensor(4, 256, dtype=e4m3), tensor(128, 256, dtype=e4m3), tensor(1, 2, dtype=f32)
    return {"quantize": (hv.hv_fp8_quantize, dict(x=x, out=q, scales=s)),
            "rms_norm": (hv.hv_fp8_rms_norm, dict(x=x, weight=w, eps=1e-6, residual=tensor(4, 256), out=q, scales=s,
                                                  residual_out=tensor(4, 256))),
            "gated": (hv.hv_fp8_gated, dict(gate=x, up=tensor(4, 256), out=q, scales=s)),
            "matmul": (hv.hv_fp8_matmul, dict(a=q, a_scales=s, b=b, b_scales=sb, out=tensor(4, 128)))}


class Library:
    """Stands in for libhv.so: notes each operator's call, the device that is current then and its stream."""

    def __init__(self, monkeypatch, current=0):
        self.calls, self.current = [], current
        monkeypatch.setattr(hv, "lib", self)
        monkeypatch.setattr(hv, "_current_device", lambda: self.current, raising=False)
        monkeypatch.setattr(hv, "_current_stream", lambda index: 1000 + index)
        monkeypatch.setattr(torch.cuda, "device", self._device)

    @contextlib.contextmanager
    def _device(self, device):
        before, self.current = self.current, torch.device(device).index
        yield
        self.current = before

    def hv_fp8_matmul_workspace_bytes(self, *args):
        return 0

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, self.current, args[-1]))
            return hv.HV_OK
        return call


@pytest.mark.parametrize("operator", OPERATORS)
@pytest.mark.parametrize("current", [0, 1])
def test_the_tensors_gpu_is_current_for_the_call(monkeypatch, operator, current):
    """A stream's handle of zero means the current device's default stream, so a call on another device's tensors
    would run there, out of order with their own stream."""
    library = Library(monkeypatch, current)
    call, args = arguments()[operator]
    call(**args)
    assert library.calls == [("hv_fp8_" + operator, 1, 1001)]
    assert library.current == current


# --------------------------------------------------------------------------
# scratch

@pytest.fixture
def streams(monkeypatch):
    """The current stream's handle and whether it is being captured, to be set by the test."""
    now = {"stream": 7, "capturing": False}
    monkeypatch.setattr(hv, "_current_device", lambda: 0)
    monkeypatch.setattr(hv, "_current_stream", lambda index: now["stream"])
    monkeypatch.setattr(hv, "_capturing", lambda: now["capturing"], raising=False)
    return now


def test_each_stream_has_scratch_of_its_own(streams):
    ws = hv.Workspace("cpu")
    first = ws.get(1000)
    assert first.numel() >= 1000 and ws.get(500) is first
    streams["stream"] = 8  # its calls may run beside those of the first
    second = ws.get(1000)
    assert second.data_ptr() != first.data_ptr()
    streams["stream"] = 7
    assert ws.get(1000) is first
    assert ws.get(5000).numel() >= 5000 and ws.get(1000).numel() >= 5000


def test_scratch_that_a_capture_was_given_stays(streams):
    """A graph's replays write there for as long as the graph lives, whatever is called in between."""
    ws = hv.Workspace("cpu")
    eager = ws.get(1000)
    streams["capturing"] = True
    buffers = [ws.get(1000), ws.get(3000)]
    kept = [weakref.ref(b) for b in buffers]
    addresses = [b.data_ptr() for b in buffers]
    del buffers
    streams["capturing"] = False
    assert ws.get(1000) is eager and eager.data_ptr() not in addresses  # eager calls may run beside a replay
    ws.get(1 << 20)
    streams["capturing"] = True
    ws.get(1 << 21)
    gc.collect()
    assert all(k() is not None for k in kept)


@pytest.mark.parametrize("device", ["cpu", "cuda:0"])
def test_scratch_elsewhere_is_refused(monkeypatch, device):
    library = Library(monkeypatch, 1)
    library.hv_fp8_matmul_workspace_bytes = lambda *args: 4096
    monkeypatch.setattr(hv.Workspace, "get", lambda self, nbytes: torch.empty(nbytes, dtype=torch.uint8))
    call, args = arguments()["matmul"]
    with pytest.raises(ValueError, match="workspace"):
        call(**args, workspace=hv.Workspace(device))
    assert library.calls == []


# --------------------------------------------------------------------------
# gradients

@pytest.mark.parametrize("operator", OPERATORS)
def test_gradients_are_refused_where_they_would_be_lost(monkeypatch, operator):
    """No backward pass: a call that autograd records is refused, and runs where nothing is recorded."""
    library = Library(monkeypatch, 1)
    call, args = arguments()[operator]
    wide = [k for k, v in args.items() if isinstance(v, torch.Tensor) and v.dtype in (torch.bfloat16, torch.float32)]
    for name in wide:
        args = arguments()[operator][1]
        args[name].requires_grad_()
        with pytest.raises(ValueError, match=f"{name} requires a gradient"):
            call(**args)
        assert library.calls == []
        with torch.no_grad():
            call(**args)
        assert len(library.calls) == 1
        library.calls.clear()
