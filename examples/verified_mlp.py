"""A decoder's MLP on weights held in 8 bits that are verified where they are used.

1. The projections of one layer are quantised on the GPU (codes and scales).
2. Their bytes, exactly as the product reads them, are the messages of a
   manifest root; a publisher would sign it, here it is kept.
3. The layer refuses to run until the bytes match that root.
4. Prefill and decode run norm, product, gate and product on them, decode beside a
   monitor that keeps rehashing the same bytes on a stream of its own.

    python examples/verified_mlp.py                     # the 70B shape: d 8192, FFN 28672
    python examples/verified_mlp.py --d 512 --ffn 1024  # small
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2510_23938_amd import hv  # noqa: E402

CHUNK = 64 << 10
EPS = 1e-5


class VerifiedMLP:
    """silu(norm(x + residual) Wg) * (norm(x + residual) Wu) Wd, on 8-bit weights under a manifest root."""

    def __init__(self, norm, gate_up, down, expected: bytes):
        """``gate_up`` [2 ffn, d] and ``down`` [d, ffn]: (codes, scales) by blocks; ``expected``: their root."""
        for codes, _ in (gate_up, down):
            if codes.stride(0) % 16 or codes.data_ptr() % 16:  # a product may copy such rows before it reads them
                raise ValueError("rows that are not 16-byte aligned would not be multiplied where they were verified")
        self.norm, self.gate_up, self.down = norm, gate_up, down
        self.pipe = hv.Pipeline(self.messages(norm, gate_up, down), CHUNK)
        if not self.pipe.run(expected):
            raise hv.VerificationError("the layer's bytes differ from what was published")
        self.workspace = hv.Workspace(norm.device)

    @staticmethod
    def messages(norm, gate_up, down):
        """The layer's bytes in a fixed order: what is hashed is what the products read."""
        return [norm, *gate_up, *down]

    @classmethod
    def root_of(cls, norm, gate_up, down) -> bytes:
        """The manifest root a publisher signs."""
        return bytes(hv.Pipeline(cls.messages(norm, gate_up, down), CHUNK).compute().cpu().numpy().reshape(-1))

    def __call__(self, x, residual):
        """(output [tokens, d], the residual of the next layer)."""
        codes, scales, h = hv.hv_fp8_rms_norm(x, self.norm, EPS, residual=residual)
        both = hv.hv_fp8_matmul(codes, scales, *self.gate_up, x.dtype, workspace=self.workspace)
        ffn = both.shape[1] // 2
        codes, scales = hv.hv_fp8_gated(both[:, :ffn], both[:, ffn:])
        return hv.hv_fp8_matmul(codes, scales, *self.down, x.dtype, workspace=self.workspace), h

    def monitor(self, stream=None):
        """Rehashes the layer's bytes against the digests of the verification above."""
        return hv.Monitor(self.pipe.keepalive, CHUNK, self.pipe.leaves, stream=stream)


def weights(d: int, ffn: int, device, seed: int = 1):
    """(norm, gate and up as one matrix, down): random weights of a decoder's shape, the matrices in 8 bits."""
    gen = torch.Generator(device=device).manual_seed(seed)

    def matrix(rows, cols):
        return torch.randn(rows, cols, generator=gen, device=device, dtype=torch.bfloat16) * 0.02

    norm = (1 + 0.1 * torch.randn(d, generator=gen, device=device)).to(torch.bfloat16)
    return norm, hv.hv_fp8_quantize(matrix(2 * ffn, d), "blocks"), hv.hv_fp8_quantize(matrix(d, ffn), "blocks")


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--d", type=int, default=8192)
    ap.add_argument("--ffn", type=int, default=28672)
    ap.add_argument("--prefill", type=int, default=2048, help="tokens of a prefill")
    ap.add_argument("--decode", type=int, default=8, help="sequences decoding")
    ap.add_argument("--steps", type=int, default=20)
    args = ap.parse_args(argv)
    dev = torch.device("cuda", torch.cuda.current_device())

    layer = weights(args.d, args.ffn, dev)
    root = VerifiedMLP.root_of(*layer)
    nbytes = sum(t.numel() * t.element_size() for t in VerifiedMLP.messages(*layer))
    mlp = VerifiedMLP(*layer, root)
    print(f"verified {nbytes / 1e6:.1f} MB of codes and scales, root {root.hex()[:16]}...")

    def inputs(tokens):
        return (torch.randn(tokens, args.d, device=dev, dtype=torch.bfloat16) for _ in range(2))

    def timed(x, r, first=lambda: None):
        mlp(x, r)
        torch.cuda.synchronize(dev)
        first()
        t = time.perf_counter()
        for _ in range(args.steps):
            y, _ = mlp(x, r)
        torch.cuda.current_stream(dev).synchronize()  # this stream's work only
        t = time.perf_counter() - t
        assert bool(torch.isfinite(y).all())
        return t / args.steps

    flops = 6 * args.d * args.ffn
    s = timed(*inputs(args.prefill))
    print(f"prefill of {args.prefill} tokens: {s * 1e6:.0f} us, {flops * args.prefill / s / 1e12:.0f} TFLOP/s")
    s = timed(*inputs(args.decode))
    print(f"decode of {args.decode} sequences: {s * 1e6:.0f} us, {nbytes / s / 1e9:.0f} GB/s of weights")

    mon = mlp.monitor()
    s = timed(*inputs(args.decode), mon.sweep)  # its scans are in flight beside the decode steps
    still = "still" if not mon.stream.query() else "no longer"
    mon.poll(wait=True)
    print(f"decode beside the monitor ({still} at work at the end): {s * 1e6:.0f} us; changed chunks: {mon.mismatches}")
    layer[1][0].view(torch.uint8)[0, 0] ^= 1  # one bit of one code
    torch.cuda.synchronize(dev)
    mon.sweep()
    mon.poll(wait=True)
    print(f"after one flipped bit, changed chunks (leaf, count, first, length): {mon.mismatches}")
    try:
        VerifiedMLP(*layer, root)
    except hv.VerificationError as e:
        print("loading it again:", e)


if __name__ == "__main__":
    main()
