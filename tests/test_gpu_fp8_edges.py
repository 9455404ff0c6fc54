"""The 8-bit operators at the ends of their ranges, against their definitions in 64 bits (oracle/fp8.py), and
their calls on other streams, with shared scratch and with rows far apart."""
import ctypes
import importlib.util
import os

import numpy as np
import pytest
import torch

import test_gpu_fp8 as base
from conftest import ROOT
from oracle import fp8
from paper_2510_23938_amd import hv  # noqa: E402  (a missing library fails the run, never skips it)

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda")
TYPES = base.TYPES


@pytest.mark.parametrize("dtype", TYPES)
def test_gated_by_a_closing_gate(dtype):
    """exp(-gate) leaves 32 bits at -88.7, and its reciprocal is subnormal from -87.3 on, while the gate's product
    with a large factor is an ordinary number.  Two exponentials of half the gate, each within an ulp, and three
    products stay below the bound on y's relative error."""
    up = 6e4 if dtype == "f16" else 1e36
    last = -96 if dtype == "f16" else -150  # y stays above the smallest scale's 448
    gate = np.linspace(-80, last, 12)[:, None] + np.linspace(0, 3, 300)[None, :]  # groups of neighbouring gates
    mixed = np.linspace(last, 4, 300)[None, :] * np.ones((4, 1))                  # and of all
    rng = np.random.default_rng(21)
    g = base.on_gpu(np.concatenate([gate, mixed]), TYPES[dtype])
    u = base.on_gpu(up * rng.uniform(0.25, 1, (16, 300)) * rng.choice([-1, 1], (16, 300)), TYPES[dtype])
    codes, scales = hv.hv_fp8_gated(g, u)
    y = fp8.gated(g.double().cpu().numpy(), u.double().cpu().numpy())
    got = scales.cpu().numpy()
    want = fp8.group_scales(y, 1)
    assert (want > 2.0 ** -126).all()
    assert np.all(np.abs(got / want - 1) <= base.Y_ERROR)
    base.check_codes(base.bytes_of(codes), y, got, 1, 2 * base.Y_ERROR)


def test_matmul_scratch_of_a_graph_survives_larger_calls():
    """A product whose columns are split, captured; a larger one on the same workspace outgrows the scratch; what is
    allocated then is not written by the graph's replays, and their results stay right."""
    rng = np.random.default_rng(23)
    small, large = base.operands(rng, 40, 300, 9000)[1], base.operands(rng, 100, 600, 20000)[1]
    need = hv.lib.hv_fp8_matmul_workspace_bytes(hv.HV_BF16, 0, 40, 300, 9000)
    more = hv.lib.hv_fp8_matmul_workspace_bytes(hv.HV_BF16, 1, 100, 600, 20000)  # 20000 is a multiple of 16
    assert 0 < need < more
    ws = hv.Workspace(DEV)
    side = torch.cuda.Stream(DEV)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = hv.hv_fp8_matmul(*small, workspace=ws).clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = hv.hv_fp8_matmul(*small, workspace=ws)
        wanted_large = hv.hv_fp8_matmul(*large)
        canaries = []
        for _ in range(3):
            assert torch.equal(hv.hv_fp8_matmul(*large, workspace=ws), wanted_large)
            canaries += [torch.full((need,), 0x55, dtype=torch.uint8, device=DEV) for _ in range(8)]
            got.zero_()
            graph.replay()
            side.synchronize()
            assert torch.equal(got, want)
            assert all(bool((c == 0x55).all()) for c in canaries)


def test_matmul_on_two_streams_with_one_workspace():
    """Each stream's calls have scratch of their own: products that run at once do not mix their parts' sums."""
    rng = np.random.default_rng(24)
    operands = [base.operands(rng, 40, 300, 9000)[1] for _ in range(2)]
    want = [hv.hv_fp8_matmul(*o) for o in operands]
    ws = hv.Workspace(DEV)
    streams = [torch.cuda.Stream(DEV) for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[i].append(hv.hv_fp8_matmul(*operands[i], workspace=ws))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(g, want[i]) for g in got[i])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_matmul_of_rows_far_apart_needs_no_workspace(dtype):
    """Rows of 2^23 bytes or more apart go straight from memory, whatever the sizes: no sums to join, no copies."""
    m, n, k = 40, 300, 9000
    host, gpu = base.operands(np.random.default_rng(22), m, n, k, near=dtype != "f32")
    assert hv.lib.hv_fp8_matmul_workspace_bytes(hv.TYPES[TYPES[dtype]], 1, m, n, k) > 0  # for rows nearer by
    ld = 1 << 23

    def apart(t):
        wide = torch.empty(t.shape[0], ld, dtype=torch.uint8, device=DEV)[:, :k].view(torch.float8_e4m3fn)
        wide.view(torch.uint8).copy_(t.view(torch.uint8))
        return wide

    a, sa, b, sb = apart(gpu[0]), gpu[1], apart(gpu[2]), gpu[3]
    out = torch.empty(m, n, dtype=TYPES[dtype], device=DEV)
    st = hv.lib.hv_fp8_matmul(hv.TYPES[TYPES[dtype]], a.data_ptr(), ld, sa.data_ptr(), b.data_ptr(), ld, sb.data_ptr(),
                              m, n, k, out.data_ptr(), n, None, 0, torch.cuda.current_stream().cuda_stream)
    assert st == hv.HV_OK, hv.lib.hv_last_error()
    base.check_product(out.double().cpu().numpy(), host, dtype)


@pytest.mark.parametrize("odd", ["a", "b", "both"])
def test_matmul_copies_no_operand_whose_rows_are_aligned(odd):
    """Where the rows of one operand are at odd addresses and copying them pays, the other one, such as verified
    weights, is read where it lies: the workspace's place for its copy is not written."""
    m, n, k = 333, 11008, 1024
    assert [p[0] for p in hv.matmul_launches(m, n, k, torch.bfloat16, False)] == ["pack", "192x128"]
    host, (a, sa, b, sb) = base.operands(np.random.default_rng(25), m, n, k, near=True)

    def moved(t):  # its first code one byte past an aligned address
        return base.codes_on_gpu(t.view(torch.uint8).cpu().numpy(), 0, 1)

    a = moved(a) if odd != "b" else a
    b = moved(b) if odd != "a" else b
    out = torch.empty(m, n, dtype=torch.bfloat16, device=DEV)
    size = hv.lib.hv_fp8_matmul_workspace_bytes(hv.HV_BF16, 0, m, n, k)
    ws = torch.full((size,), 0x55, dtype=torch.uint8, device=DEV)
    st = hv.lib.hv_fp8_matmul(hv.HV_BF16, a.data_ptr(), k, sa.data_ptr(), b.data_ptr(), k, sb.data_ptr(), m, n, k,
                              out.data_ptr(), n, ws.data_ptr(), size, torch.cuda.current_stream().cuda_stream)
    assert st == hv.HV_OK, hv.lib.hv_last_error()
    base.check_product(out.double().cpu().numpy(), host, "bf16")
    place = {"a": ws[:m * k].view(m, k), "b": ws[m * k + -(m * k) % 256:][:n * k].view(n, k)}
    for name, t in (("a", a), ("b", b)):
        if odd in (name, "both"):
            assert torch.equal(place[name], t.view(torch.uint8))
        else:
            assert bool((place[name] == 0x55).all())


def test_verified_layer_refuses_weights_that_a_product_would_copy():
    spec = importlib.util.spec_from_file_location("verified_mlp", os.path.join(ROOT, "examples", "verified_mlp.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    layer = example.weights(256, 384, DEV)
    root = example.VerifiedMLP.root_of(*layer)
    example.VerifiedMLP(*layer, root)
    for d, ffn in ((250, 384), (256, 392)):  # rows of a length that is no multiple of 16
        odd = example.weights(d, ffn, DEV)
        with pytest.raises(ValueError, match="16-byte"):
            example.VerifiedMLP(*odd, example.VerifiedMLP.root_of(*odd))
    norm, (codes, scales), down = layer
    moved = torch.empty(codes.numel() + 1, dtype=torch.uint8, device=DEV)[1:].view(codes.shape)
    moved.copy_(codes.view(torch.uint8))
    with pytest.raises(ValueError, match="16-byte"):
        example.VerifiedMLP(norm, (moved.view(codes.dtype), scales), down, root)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fragments", [1, 2, 3, 4, 5, 7])
def test_matmul_by_each_number_of_fragments(fragments, dtype):
    """Up to 16 rows of A against each number of fragments of B a workgroup, the last workgroup's not all there."""
    kind = {1: 1, 2: 2, 3: 14, 4: 3, 5: 15, 7: 4}[fragments]
    for m, short, k, pad in ((16, 0, 300, 4), (16, 27, 1024, 0), (15, 19, 300, 20)):
        n = 4096 * fragments - short
        assert _kinds(m, n, k, dtype) == [kind]
        base.product(m, n, k, dtype, pad)


def _kinds(m, n, k, dtype):
    count = ctypes.c_int(0)
    kind, splits = (ctypes.c_int * 3)(), (ctypes.c_uint32 * 3)()
    rows, cols = (ctypes.c_uint64 * 3)(), (ctypes.c_uint64 * 3)()
    assert hv.lib.hv_fp8_matmul_launches(hv.TYPES[TYPES[dtype]], 1, m, n, k, ctypes.byref(count), kind, rows, cols,
                                         splits) == hv.HV_OK
    return list(kind[:count.value])
