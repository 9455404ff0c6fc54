"""The 8-bit operators whose time is watched: what a program that serves
verified weights held in 8 bits asks of this library.

A case is a dict of plain values.  ``op`` names the operator:

* ``matmul``    A [m, k] times the transpose of B [n, k], both in 8-bit floating
  point (e4m3), A with a scale for every 128 columns of a row, B with one for
  every block of 128 x 128;
* ``rms_norm``  the residual's addition, root-mean-square norm and the output in
  8 bits with a scale for every 128 columns of a row;
* ``gated``     silu(gate) * up with the same kind of output;
* ``quantize``  a matrix to 8 bits, scales by rows (activations) or blocks (weights).

``pad`` is how many elements lie between the rows of an input.  The plain forms
work in 32 bits and round once; where a group of 128 is all zeros its scale is 1.
"""
import math

import torch

own = False

GROUP = 128
LARGEST = 448.0  # of e4m3
SMALLEST_SCALE = 2.0 ** -126
EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
MOST_FLOPS = 2 * 2048 * 28672 * 8192  # of a drawn product: the largest listed one
MOST_ELEMENTS = 16384 * 8192          # of a drawn matrix of the other operators


def _matmul(m, n, k, dtype, pad=0):
    return {"op": "matmul", "m": m, "n": n, "k": k, "type": dtype, "pad": pad}


def _norm(rows, width, dtype, residual, pad=0):
    return {"op": "rms_norm", "rows": rows, "width": width, "type": dtype, "residual": residual, "pad": pad}


def _gated(rows, width, dtype, joint):
    return {"op": "gated", "rows": rows, "width": width, "type": dtype, "joint": joint}


def _quantize(rows, width, dtype, tile, pad=0):
    return {"op": "quantize", "rows": rows, "width": width, "type": dtype, "tile": tile, "pad": pad}


def listed():
    return [
        # one sequence decoding: a token through an attention output projection of the 70B shape
        {"name": "token_product", **_matmul(1, 8192, 8192, "bf16")},
        # eight sequences decoding: their tokens through an up projection of the 70B shape
        {"name": "decode_product", **_matmul(8, 28672, 8192, "bf16")},
        # a short prompt through an up projection of the 7B shape
        {"name": "prompt_product", **_matmul(333, 11008, 4096, "f16")},
        # a prefill of 2048 tokens through an up projection of the 70B shape
        {"name": "prefill_product", **_matmul(2048, 28672, 8192, "bf16")},
        # a head pruned to odd sizes, its logits in 32 bits, rows at odd addresses
        {"name": "odd_product", **_matmul(77, 5001, 4093, "f32", 3)},
        # the norm ahead of each projection, one token
        {"name": "token_norm", **_norm(1, 8192, "bf16", True)},
        # the same for a batch of prompts
        {"name": "prefill_norm", **_norm(16384, 8192, "bf16", True)},
        # a first norm (no residual yet) on columns of a wider matrix in 32 bits
        {"name": "odd_norm", **_norm(1001, 4095, "f32", False, 33)},
        # between the products of an MLP of the 70B shape: eight tokens, then a prefill whose
        # gate and up came from one product
        {"name": "decode_gated", **_gated(8, 28672, "bf16", False)},
        {"name": "prefill_gated", **_gated(2048, 28672, "bf16", True)},
        # a projection of the 70B shape to 8 bits, before it is hashed
        {"name": "quantize_weight", **_quantize(28672, 8192, "bf16", "blocks")},
        # attention's output to 8 bits, ragged
        {"name": "quantize_rows", **_quantize(1777, 4104, "f16", "rows", 8)},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """Spread over the logarithm; every other one a multiple of the group."""
    v = _spread(rng, lo, hi)
    return max(GROUP, v // GROUP * GROUP) if rng.random() < 0.5 else v


def draw(rng):
    op = rng.choice(["matmul", "matmul", "rms_norm", "gated", "quantize"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "matmul":
        n, k = _size(rng, 64, 57344), _size(rng, 64, 28672)
        m = _spread(rng, 1, 4096)
        m = max(1, min(m, MOST_FLOPS // (2 * n * k)))
        return _matmul(m, n, k, dtype, rng.choice([0, 0, 16, 5]))
    width = _size(rng, 64, 32768)
    rows = max(1, min(_spread(rng, 1, 65536), MOST_ELEMENTS // (width * BYTES[dtype] // 2)))
    pad = rng.choice([0, 0, 8, 7])
    if op == "rms_norm":
        return _norm(rows, width, dtype, rng.random() < 0.7, pad)
    if op == "gated":
        return _gated(max(1, rows // 2), width, dtype, rng.random() < 0.5)
    return _quantize(rows, width, dtype, rng.choice(["rows", "blocks"]), pad)


# --------------------------------------------------------------------------
# plain forms

def _groups(y):
    """[rows, width] as [rows, groups, 128], the last group filled up with zeros."""
    rows, width = y.shape
    full = -(-width // GROUP) * GROUP
    if full != width:
        y = torch.cat([y, y.new_zeros(rows, full - width)], 1)
    return y.view(rows, full // GROUP, GROUP)


def _scale_of(largest):
    return torch.where(largest > 0, (largest / LARGEST).clamp_min(SMALLEST_SCALE), torch.ones_like(largest))


def _finite(y):
    return torch.where(torch.isfinite(y), y.abs(), torch.zeros_like(y))


def _rows_to_8_bits(y):
    """(codes [rows, width], scales [rows, groups]) of a 32-bit matrix."""
    rows, width = y.shape
    g = _groups(y)
    scales = _scale_of(_finite(g).amax(2))
    codes = (g / scales[:, :, None]).view(rows, -1)[:, :width].contiguous().to(torch.float8_e4m3fn)
    return codes, scales


def _blocks_to_8_bits(y):
    """(codes [rows, width], scales [row groups, groups]) of a 32-bit matrix."""
    rows, width = y.shape
    g = _groups(y)
    row_groups = -(-rows // GROUP)
    largest = _finite(g).amax(2)
    if rows != row_groups * GROUP:
        largest = torch.cat([largest, largest.new_zeros(row_groups * GROUP - rows, largest.shape[1])], 0)
    scales = _scale_of(largest.view(row_groups, GROUP, -1).amax(1))
    by_row = scales.repeat_interleave(GROUP, 0)[:rows]
    codes = (g / by_row[:, :, None]).view(rows, -1)[:, :width].contiguous().to(torch.float8_e4m3fn)
    return codes, scales


def _plain_matmul(s):
    k, n = s["a"].shape[1], s["b"].shape[0]
    by_column = s["a_scales"].repeat_interleave(GROUP, 1)[:, :k]
    by_element = s["b_scales"].repeat_interleave(GROUP, 0)[:n].repeat_interleave(GROUP, 1)[:, :k]
    return torch.matmul(s["a"].float() * by_column, (s["b"].float() * by_element).t()).to(s["type"])


def _plain_norm(s):
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * s["weight"].float()
    codes, scales = _rows_to_8_bits(y)
    return (codes, scales, h.to(s["x"].dtype)) if s["residual"] is not None else (codes, scales)


def _plain_gated(s):
    g = s["gate"].float()
    return _rows_to_8_bits(g / (1 + torch.exp(-g)) * s["up"].float())


def _plain_quantize(s):
    return (_rows_to_8_bits if s["tile"] == "rows" else _blocks_to_8_bits)(s["x"].float())


# --------------------------------------------------------------------------
# inputs

def _activations(gen, rows, width, dtype, pad, dev):
    """What the layers of a decoder pass on: rows of differing size, a few columns far above the others."""
    wide = torch.randn(rows, width + pad, generator=gen, device=dev)
    wide *= torch.exp(torch.randn(rows, 1, generator=gen, device=dev) * 0.5)
    strong = torch.rand(1, width + pad, generator=gen, device=dev) < 0.002
    wide = torch.where(strong, wide * 30, wide).to(dtype)
    return wide[:, :width]


def _in_8_bits(x, tile, pad):
    codes, scales = (_rows_to_8_bits if tile == "rows" else _blocks_to_8_bits)(x.float())
    if pad:
        wide = torch.zeros(codes.shape[0], codes.shape[1] + pad, dtype=torch.uint8, device=codes.device)
        wide = wide.fill_(0x7f).view(torch.float8_e4m3fn)  # between the rows lies what nobody may read: NaN
        wide[:, :codes.shape[1]] = codes
        codes = wide[:, :codes.shape[1]]
    return codes, scales


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dtype, op = TYPES[case["type"]], case["op"]
    s = {"op": op, "type": dtype}
    if op == "matmul":
        x = _activations(gen, case["m"], case["k"], torch.bfloat16, 0, dev)
        s["a"], s["a_scales"] = _in_8_bits(x, "rows", case["pad"])
        w = torch.randn(case["n"], case["k"], generator=gen, device=dev) * 0.02
        s["b"], s["b_scales"] = _in_8_bits(w, "blocks", case["pad"])
        return s
    rows, width = case["rows"], case["width"]
    if op == "rms_norm":
        s["x"] = _activations(gen, rows, width, dtype, case["pad"], dev)
        s["residual"] = _activations(gen, rows, width, dtype, case["pad"], dev) if case["residual"] else None
        s["weight"] = (1 + 0.1 * torch.randn(width, generator=gen, device=dev)).to(dtype)
    elif op == "gated":
        if case["joint"]:
            both = _activations(gen, rows, 2 * width, dtype, 0, dev)
            s["gate"], s["up"] = both[:, :width], both[:, width:]
        else:
            s["gate"] = _activations(gen, rows, width, dtype, 0, dev)
            s["up"] = _activations(gen, rows, width, dtype, 0, dev)
    else:
        s["tile"] = case["tile"]
        s["x"] = _activations(gen, rows, width, dtype, case["pad"], dev)
        if case["tile"] == "blocks":
            s["x"] *= 0.02
    return s


def run(s):
    if not own:
        return {"matmul": _plain_matmul, "rms_norm": _plain_norm, "gated": _plain_gated,
                "quantize": _plain_quantize}[s["op"]](s)
    from paper_2510_23938_amd import hv
    if s["op"] == "matmul":
        return hv.hv_fp8_matmul(s["a"], s["a_scales"], s["b"], s["b_scales"], s["type"])
    if s["op"] == "rms_norm":
        codes, scales, h = hv.hv_fp8_rms_norm(s["x"], s["weight"], EPS, residual=s["residual"])
        return (codes, scales, h) if h is not None else (codes, scales)
    if s["op"] == "gated":
        return hv.hv_fp8_gated(s["gate"], s["up"])
    return hv.hv_fp8_quantize(s["x"], s["tile"])


def work(case):
    e = BYTES[case["type"]]
    if case["op"] == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        kg = -(-k // GROUP)
        return {"bytes": m * k + n * k + 4 * kg * (m + -(-n // GROUP)) + m * n * e, "flops": 2 * m * n * k}
    r, w = case["rows"], case["width"]
    groups = -(-w // GROUP)
    if case["op"] == "rms_norm":
        moved = 3 if case["residual"] else 1  # x alone, or x and the residual read and their sum written
        return {"bytes": r * w * (moved * e + 1) + w * e + 4 * r * groups, "flops": 8 * r * w}
    if case["op"] == "gated":
        return {"bytes": r * w * (2 * e + 1) + 4 * r * groups, "flops": 8 * r * w}
    scales = groups * (r if case["tile"] == "rows" else -(-r // GROUP))
    return {"bytes": r * w * (e + 1) + 4 * scales, "flops": 3 * r * w}


def exact(case, seed):
    """The operators from their definitions in 64 bits.  In the place of 8-bit codes stand the quotients before their
    rounding, so that a side's distance is the rounding that the format asks for and whatever it adds to that."""
    s = prepare(case, seed)
    if s["op"] == "matmul":
        a, b = s["a"].float().double(), s["b"].float().double()
        sa, sb = s["a_scales"].double(), s["b_scales"].double()
        total = torch.zeros(a.shape[0], b.shape[0], dtype=torch.float64, device=a.device)
        for g in range(sa.shape[1]):
            part = a[:, g * GROUP:(g + 1) * GROUP].contiguous() @ b[:, g * GROUP:(g + 1) * GROUP].t().contiguous()
            column = torch.arange(b.shape[0], device=a.device) // GROUP
            total += part * (sa[:, g].unsqueeze(1) * sb[column, g].unsqueeze(0))
        return total
    kept = None
    if s["op"] == "rms_norm":
        y = s["x"].double()
        if s["residual"] is not None:
            y = y + s["residual"].double()
            kept = y
        power = (y * y).sum(1) / y.shape[1]
        y = y / torch.sqrt(power + EPS)[:, None] * s["weight"].double()
    elif s["op"] == "gated":
        y = s["gate"].double() * torch.sigmoid(s["gate"].double()) * s["up"].double()
    else:
        y = s["x"].double()
    rows, width = y.shape
    high = 1 if s["op"] != "quantize" or s["tile"] == "rows" else GROUP
    scales = torch.ones(-(-rows // high), -(-width // GROUP), dtype=torch.float64, device=y.device)
    quotients = torch.empty_like(y)
    for g in range(scales.shape[1]):
        part = y[:, g * GROUP:(g + 1) * GROUP]
        largest = part.abs().amax(1)
        band = torch.arange(rows, device=y.device) // high
        top = torch.zeros(scales.shape[0], dtype=torch.float64, device=y.device)
        top = top.scatter_reduce(0, band, largest, "amax")
        scales[:, g] = torch.where(top > 0, top / LARGEST, torch.ones_like(top))
        quotients[:, g * GROUP:(g + 1) * GROUP] = part / scales[band, g][:, None]
    return (quotients, scales, kept) if kept is not None else (quotients, scales)
