"""examples/verified_mlp.py: the 8-bit operators and the verification together, on a small layer.

The layer's output against its formula in 64 bits on the same 8-bit weights.  What lies between are
the two roundings of activations to 8 bits, each a relative error of up to 2^-4 and 2.6% on average
(uniform in a binade's spacing), and bfloat16's: a product averages independent errors to
the same relative size, so two roundings give 3.7%, the gate's product of two rounded factors 5.2% in all; 8% is
allowed."""
import importlib.util
import os

import numpy as np
import pytest
import torch

from conftest import ROOT
from oracle import fp8
from paper_2510_23938_amd import hv  # noqa: E402  (a missing library fails the run, never skips it)

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda", 0)


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("verified_mlp", os.path.join(ROOT, "examples", "verified_mlp.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def numbers(codes, scales):
    c = codes.view(torch.uint8).cpu().numpy()
    return fp8.VALUES[c] * fp8.spread(scales.cpu().numpy(), 128, *c.shape)


@pytest.mark.parametrize("tokens", [1, 8, 70])
def test_layer_against_its_formula(example, tokens):
    d, ffn = 384, 640
    layer = example.weights(d, ffn, DEV)
    mlp = example.VerifiedMLP(*layer, example.VerifiedMLP.root_of(*layer))
    gen = torch.Generator(device=DEV).manual_seed(3)
    x, r = (torch.randn(tokens, d, generator=gen, device=DEV).to(torch.bfloat16) for _ in range(2))
    y, h = mlp(x, r)
    norm, want_h = fp8.rms_norm(x.float().cpu().numpy(), r.float().cpu().numpy(), layer[0].double().cpu().numpy(),
                                example.EPS)
    both = norm @ numbers(*layer[1]).T
    want = fp8.gated(both[:, :ffn], both[:, ffn:]) @ numbers(*layer[2]).T
    got = y.double().cpu().numpy()
    assert np.linalg.norm(got - want) <= 0.08 * np.linalg.norm(want)
    assert torch.equal(h.cpu(), torch.from_numpy(want_h).to(torch.bfloat16))


def test_changed_bytes_are_refused_and_seen(example):
    layer = example.weights(256, 384, DEV)
    root = example.VerifiedMLP.root_of(*layer)
    mlp = example.VerifiedMLP(*layer, root)
    mon = mlp.monitor()
    mon.sweep()
    mon.poll(wait=True)
    assert mon.mismatches == []
    for t in (layer[0].view(torch.uint8), layer[1][0].view(torch.uint8), layer[1][1].view(torch.uint8),
              layer[2][1].view(torch.uint8)):  # norm, codes and scales are all under the root
        t.view(-1)[7] ^= 4
        with pytest.raises(hv.VerificationError):
            example.VerifiedMLP(*layer, root)
        t.view(-1)[7] ^= 4
    example.VerifiedMLP(*layer, root)
    layer[2][0].view(torch.uint8)[3, 5] ^= 1
    torch.cuda.synchronize()
    mon.sweep()
    mon.poll(wait=True)
    assert len(mon.mismatches) == 1


def test_the_command_runs(example, capsys):
    example.main(["--d", "256", "--ffn", "512", "--prefill", "100", "--decode", "3", "--steps", "2"])
    out = capsys.readouterr().out
    assert "changed chunks: []" in out and "loading it again: the layer's bytes differ" in out
