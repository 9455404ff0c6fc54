"""A decoder's attention on weights held in 8 bits that are verified where they are used, with a cache in 8 bits and an
adapter for each sequence.

1. The projections to queries, keys and values and back are quantised on the GPU; their bytes and those of the
   sequences' adapters are the messages of one manifest root.
2. The layer refuses to run until the bytes match that root.
3. Prompts go through it at once, in chunks or whole: new keys and values to the pages of each sequence, attention over
   them, every sequence's adapter beside the shared products.
4. Tokens go through it one at a time for all sequences, as one captured graph whose lengths grow on the GPU.

    python examples/verified_attention.py                                   # the 70B shape: d 8192, 64 heads on 8
    python examples/verified_attention.py --d 512 --heads 8 --kv-heads 2    # small
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
PAGE = 64  # tokens of a page


class VerifiedAttention:
    """Attention of norm(x + residual), its projections on 8-bit weights and adapters under a manifest root."""

    def __init__(self, norm, qkv, out, qkv_adapters, out_adapters, heads, kv_heads, expected: bytes):
        """``qkv`` [(heads + 2 kv_heads) head_dim, d] and ``out`` [d, heads head_dim]: (codes, scales) by blocks; the
        adapters (down, up); ``expected``: the root of all their bytes."""
        self.norm, self.qkv, self.out = norm, qkv, out
        self.adapters = qkv_adapters, out_adapters
        self.heads, self.kv_heads = heads, kv_heads
        self.pipe = hv.Pipeline(self.messages(norm, qkv, out, qkv_adapters, out_adapters), CHUNK)
        if not self.pipe.run(expected):
            raise hv.VerificationError("the layer's bytes differ from what was published")
        self.workspace = hv.Workspace(norm.device)

    @staticmethod
    def messages(norm, qkv, out, qkv_adapters, out_adapters, *_):
        return [norm, *qkv, *out, *qkv_adapters, *out_adapters]

    @classmethod
    def root_of(cls, *layer) -> bytes:
        """The manifest root a publisher signs."""
        return bytes(hv.Pipeline(cls.messages(*layer), CHUNK).compute().cpu().numpy().reshape(-1))

    def __call__(self, x, residual, cache, starts, lengths, pages, adapter):
        """(output [tokens, d], the residual of the next layer); ``adapter`` [tokens] int32, -1 for none."""
        codes, scales, h = hv.hv_fp8_rms_norm(x, self.norm, EPS, residual=residual)
        rows = hv.hv_fp8_matmul(codes, scales, *self.qkv, x.dtype, workspace=self.workspace)
        hv.hv_fp8_adapters(rows, codes, scales, *self.adapters[0], adapter, out=rows, workspace=self.workspace)
        rows = rows.view(len(x), self.heads + 2 * self.kv_heads, -1)
        q, k, v = rows.split([self.heads, self.kv_heads, self.kv_heads], 1)
        hv.hv_fp8_cache_write(cache, k, v, starts, lengths, pages)
        a = hv.hv_fp8_attention(q, cache, starts, lengths, pages, workspace=self.workspace)
        codes, scales = hv.hv_fp8_quantize(a.view(len(x), -1))
        y = hv.hv_fp8_matmul(codes, scales, *self.out, x.dtype, workspace=self.workspace)
        return hv.hv_fp8_adapters(y, codes, scales, *self.adapters[1], adapter, out=y, workspace=self.workspace), h


def weights(d, heads, kv_heads, head_dim, adapters, rank, device, seed: int = 1):
    """(norm, qkv, out, adapters of both, heads, kv_heads): random weights of a decoder's shape."""
    gen = torch.Generator(device=device).manual_seed(seed)

    def matrix(*shape):
        return torch.randn(*shape, generator=gen, device=device, dtype=torch.bfloat16) * 0.02

    norm = (1 + 0.1 * torch.randn(d, generator=gen, device=device)).to(torch.bfloat16)
    width = (heads + 2 * kv_heads) * head_dim
    return (norm, hv.hv_fp8_quantize(matrix(width, d), "blocks"), hv.hv_fp8_quantize(matrix(d, heads * head_dim), "blocks"),
            (matrix(adapters, rank, d), matrix(adapters, width, rank)),
            (matrix(adapters, rank, heads * head_dim), matrix(adapters, d, rank)), heads, kv_heads)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--d", type=int, default=8192)
    ap.add_argument("--heads", type=int, default=64)
    ap.add_argument("--kv-heads", type=int, default=8)
    ap.add_argument("--head-dim", type=int, default=128)
    ap.add_argument("--rank", type=int, default=16)
    ap.add_argument("--sequences", type=int, default=8)
    ap.add_argument("--prompt", type=int, default=2048, help="tokens of a sequence's prompt")
    ap.add_argument("--steps", type=int, default=20, help="tokens after it")
    args = ap.parse_args(argv)
    dev = torch.device("cuda", torch.cuda.current_device())
    n = args.sequences

    parts = weights(args.d, args.heads, args.kv_heads, args.head_dim, n, args.rank, dev)
    layer = VerifiedAttention(*parts, VerifiedAttention.root_of(*parts))
    columns = -(-(args.prompt + args.steps + 2) // PAGE)
    cache = hv.Fp8Cache.empty(n * columns, args.kv_heads, PAGE, args.head_dim, dev)
    pages = torch.randperm(n * columns, device=dev).to(torch.int32).view(n, columns)

    def inputs(tokens):
        return [torch.randn(tokens, args.d, device=dev, dtype=torch.bfloat16) for _ in range(2)]

    sequence = torch.arange(n, dtype=torch.int32, device=dev)
    lengths = torch.full((n,), args.prompt, dtype=torch.int32, device=dev)
    prompt = (*inputs(n * args.prompt), cache, torch.arange(n + 1, dtype=torch.int32, device=dev) * args.prompt, lengths, pages,
              sequence.repeat_interleave(args.prompt))
    layer(*prompt)
    torch.cuda.synchronize(dev)
    t = time.perf_counter()
    y, _ = layer(*prompt)
    torch.cuda.synchronize(dev)
    t = time.perf_counter() - t
    assert bool(torch.isfinite(y).all())
    print(f"{n} prompts of {args.prompt} tokens: {t * 1e6:.0f} us")

    token = (*inputs(n), cache, torch.arange(n + 1, dtype=torch.int32, device=dev), lengths, pages, sequence)
    lengths += 1
    side = torch.cuda.Stream(dev)
    side.wait_stream(torch.cuda.current_stream(dev))
    with torch.cuda.stream(side):
        layer(*token)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            lengths += 1  # on the GPU, by each replay
            y, _ = layer(*token)
        side.synchronize()
        t = time.perf_counter()
        for _ in range(args.steps):
            graph.replay()
        side.synchronize()
        t = (time.perf_counter() - t) / args.steps
    assert bool(torch.isfinite(y).all()) and lengths.tolist() == [args.prompt + 1 + args.steps] * n
    print(f"a token of each of {n} sequences: {t * 1e6:.0f} us a step, at {args.prompt + 1 + args.steps} tokens in the end")


if __name__ == "__main__":
    main()
