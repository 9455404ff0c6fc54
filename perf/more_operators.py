"""The operators between and beside the projections of a decoder served on 8-bit weights, whose time is watched.

A case is a dict of plain values.  ``op`` names the operator:

* ``write``      new tokens' keys and values into pages of an 8-bit cache, a scale for
  every 16 tokens of a head;
* ``attention``  of new tokens over such a cache, causal, with shared key heads, and where asked only over a window of
  the last tokens and the first few ("sinks");
* ``adapters``   low-rank adapters of many requests at once, added to a shared projection's output: y plus, for a
  token of request i, factor[i] * (x down[i]^T) up[i]^T, with x in 8 bits as the projection took it.

A batch is ragged: sequence i has ``new`` tokens in rows starts[i] to starts[i + 1] of the inputs, which are the last
ones of its ``lengths[i]`` tokens, and its tokens lie in the pages that row i of the page table names.  The cache holds
keys as [pages, heads, page tokens, head size] and values as [pages, heads, page tokens / 16, head size, 16], 8-bit
codes (e4m3), and a power of two for each 16 tokens of a head, the smallest that keeps their codes within 448; where
a later token needs a larger one, what the 16 held before is rounded to it.
"""
import math

import torch

own = False

BLOCK = 16       # tokens of a head that share a scale
GROUP = 128      # columns of a row of 8-bit activations that share a scale
LARGEST = 448.0  # of e4m3
SMALLEST_SCALE = 2.0 ** -126
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
MOST_PAIRS = 4 * 64 * 128 * 2048 * 2049 // 2  # of a drawn attention: heads x head size x visible pairs, as the largest listed
MOST_CACHED = 64 * 8 * 128 * 5120             # of a drawn attention: cached keys' elements, as the largest listed
MOST_BYTES = 630 << 20                        # of a drawn attention
MOST_WRITTEN = 16384 * 8 * 128                # of a drawn write
MOST_ADAPTED = 2048 * 28672                   # of a drawn projection's outputs


def _write(batch, new, context, kv_heads, head, page, dtype, ragged):
    return {"op": "write", "batch": batch, "new": new, "context": context, "kv_heads": kv_heads, "head": head,
            "page": page, "type": dtype, "ragged": ragged}


def _attention(batch, new, context, heads, kv_heads, head, page, dtype, ragged, window=0, sinks=0):
    return {"op": "attention", "batch": batch, "new": new, "context": context, "heads": heads, "kv_heads": kv_heads,
            "head": head, "page": page, "type": dtype, "ragged": ragged, "window": window, "sinks": sinks}


def _adapters(requests, tokens, rank, k, n, adapters, dtype, result, without=0):
    return {"op": "adapters", "requests": requests, "tokens": tokens, "rank": rank, "k": k, "n": n,
            "adapters": adapters, "type": dtype, "result": result, "without": without}


def listed():
    return [
        # eight sequences decoding at the 70B shape: a token each into blocks that are partly filled
        {"name": "decode_write", **_write(8, 1, 1000, 8, 128, 64, "bf16", True)},
        # prompts of a prefill at the 70B shape
        {"name": "prompt_write", **_write(8, 2048, 2048, 8, 128, 64, "bf16", False)},
        # chunks of prompts of odd lengths, in the middle of blocks, odd sizes of heads and pages
        {"name": "odd_write", **_write(13, 333, 1500, 5, 80, 48, "f16", True)},
        # one sequence decoding at the 70B shape, a short context: latency
        {"name": "token_attention", **_attention(1, 1, 777, 64, 8, 128, 64, "bf16", False)},
        # a batch decoding at the 70B shape, contexts of differing lengths
        {"name": "decode_attention", **_attention(64, 1, 8192, 64, 8, 128, 64, "bf16", True)},
        # one sequence decoding behind a very long context
        {"name": "long_attention", **_attention(1, 1, 131072, 64, 8, 128, 128, "bf16", False)},
        # drafted tokens checked at once at the 7B shape, a key head for every head
        {"name": "draft_attention", **_attention(16, 5, 2500, 32, 32, 128, 16, "f16", True)},
        # a prefill of four prompts at the 70B shape
        {"name": "prefill_attention", **_attention(4, 2048, 2048, 64, 8, 128, 64, "bf16", False)},
        # a chunk of a long prompt that sees a window and the first tokens, odd sizes
        {"name": "window_attention", **_attention(1, 777, 30001, 20, 4, 80, 48, "bf16", False, 4095, 5)},
        # 32 requests decoding, each with an adapter of its own, through an output projection of the 70B shape
        {"name": "decode_adapters", **_adapters(32, 1, 16, 8192, 8192, 32, "bf16", "bf16")},
        # four prompts with adapters through an up projection of the 70B shape
        {"name": "prefill_adapters", **_adapters(4, 512, 16, 8192, 28672, 8, "bf16", "bf16")},
        # an odd rank and odd sizes, logits in 32 bits, some requests without an adapter
        {"name": "odd_adapters", **_adapters(19, 11, 13, 4093, 5001, 7, "f16", "f32", 3)},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["write", "attention", "attention", "attention", "adapters", "adapters"])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    head = rng.choice([64, 128, 128, 128, 80, 96, 16, 256, 192])
    page = rng.choice([16, 32, 64, 64, 128, 256, 48])
    ragged = rng.random() < 0.7
    if op == "write":
        batch, kv_heads = _spread(rng, 1, 256), rng.choice([1, 2, 5, 8, 8, 32])
        most = MOST_WRITTEN // (batch * kv_heads * head)
        new = 1 if rng.random() < 0.4 else max(1, min(_spread(rng, 1, 16384), most))
        context = new + (0 if rng.random() < 0.4 else rng.randrange(2000))
        return _write(batch, new, context, kv_heads, head, page, rng.choice([dtype, dtype, "f32"]), ragged)
    if op == "attention":
        kv_heads = rng.choice([1, 2, 4, 5, 8, 8, 32])
        heads = kv_heads * rng.choice([share for share in (1, 1, 2, 4, 5, 7, 8, 8, 16) if share * kv_heads <= 128])
        kind = rng.choice(["token", "token", "draft", "prompt"])
        batch = _spread(rng, 1, 256) if kind != "prompt" else _spread(rng, 1, 16)
        context = max(1, min(_spread(rng, 1, 200000), MOST_CACHED // (batch * kv_heads * head)))
        new = {"token": 1, "draft": rng.randint(2, 16), "prompt": _spread(rng, 17, 8192)}[kind]
        new = max(1, min(new, context))
        while new * context * batch * heads * head > MOST_PAIRS and new > 1:
            new = max(1, new * 3 // 4)
        window = _spread(rng, 1, 8192) if rng.random() < 0.3 else 0
        sinks = rng.choice([0, 1, 4, 70]) if window else 0
        case = _attention(batch, new, context, heads, kv_heads, head, page, dtype, ragged, window, sinks)
        while work(case)["bytes"] > MOST_BYTES:
            case["batch"] = case["batch"] * 3 // 4
        return case
    rank = rng.choice([8, 16, 16, 32, 64, 128, 4, 1, 13])
    k, n = _spread(rng, 64, 28672), _spread(rng, 64, 28672)
    if rng.random() < 0.6:
        k, n = max(GROUP, k // GROUP * GROUP), max(GROUP, n // GROUP * GROUP)
    requests = _spread(rng, 1, 128)
    most = min(MOST_ADAPTED // (n * requests), MOST_ADAPTED // (k * requests))
    tokens = 1 if rng.random() < 0.5 else max(1, min(_spread(rng, 1, 2048), most))
    adapters = rng.choice([1, 4, 16, requests])
    while adapters * rank * (k + n) > 1 << 28:
        adapters = max(1, adapters // 2)
    return _adapters(requests, tokens, rank, k, n, adapters, dtype, rng.choice([dtype, dtype, "f32"]),
                     rng.choice([0, 0, min(3, requests)]))


# --------------------------------------------------------------------------
# the batch that a case describes (by the case alone: what a pass costs goes by it)

def _lengths(case):
    """(new tokens, tokens in all) of each sequence."""
    new, context = [], []
    for i in range(case["batch"]):
        part = (i * 0.6180339887 + 0.35) % 1.0 if case["ragged"] else 1.0
        c = max(1, int(case["context"] * (0.25 + 0.75 * part)))
        n = max(1, int(case["new"] * (0.25 + 0.75 * ((i * 0.7548776662 + 0.6) % 1.0)))) if case["ragged"] else case["new"]
        new.append(min(n, c))
        context.append(c)
    return new, context


def _visible(case):
    """(cached tokens that some new token sees, pairs of a new token and one that it sees), of the whole batch."""
    seen, pairs = 0, 0
    for n, c in zip(*_lengths(case)):
        if not case["window"]:
            seen += c
            pairs += n * (c - n) + n * (n + 1) // 2
            continue
        for p in range(c - n, c):
            first = max(0, p - case["window"] + 1)
            pairs += p - first + 1 + min(first, case["sinks"])
        first = max(0, c - n - case["window"] + 1)
        seen += c - first + min(first, case["sinks"])
    return seen, pairs


def work(case):
    e = BYTES[case["type"]]
    if case["op"] == "write":
        new, context = _lengths(case)
        blocks = sum((c - 1) // BLOCK - (c - n) // BLOCK + 1 for n, c in zip(new, context))
        elements = 2 * sum(new) * case["kv_heads"] * case["head"]
        return {"bytes": elements * (e + 1) + 2 * 4 * blocks * case["kv_heads"], "flops": 2 * elements}
    if case["op"] == "attention":
        seen, pairs = _visible(case)
        rows = sum(_lengths(case)[0])
        return {"bytes": 2 * rows * case["heads"] * case["head"] * e +
                2 * seen * case["kv_heads"] * (case["head"] + 4 / BLOCK) + 4 * (seen / case["page"]),
                "flops": 4 * pairs * case["heads"] * case["head"]}
    rows = case["requests"] * case["tokens"]
    used = len({i % case["adapters"] for i in range(case["without"], case["requests"])})
    adapted = (case["requests"] - case["without"]) * case["tokens"]
    return {"bytes": adapted * (case["k"] + 4 * -(-case["k"] // GROUP)) + used * case["rank"] * (case["k"] + case["n"]) * e +
            2 * rows * case["n"] * BYTES[case["result"]] + 4 * rows,
            "flops": 2 * adapted * case["rank"] * (case["k"] + case["n"])}


# --------------------------------------------------------------------------
# inputs

def _powers(largest):
    """The smallest powers of two that keep values up to these within the format's largest, in 32 bits."""
    part, power = torch.frexp(largest.float())          # largest = part * 2^power, part in [0.5, 1); 448 = 0.875 * 2^9
    power = power - 9 + (part > 0.875).int()
    scale = torch.ldexp(torch.ones_like(largest), power.clamp_min(-126))
    return torch.where(largest > 0, scale, torch.full_like(scale, SMALLEST_SCALE))


def _pages(gen, case, dev):
    """(page table, pages of the pool): pages in any order, as they come free."""
    counts = [-(-c // case["page"]) for c in _lengths(case)[1]]
    total = sum(counts)
    pool = total + 3
    order = torch.randperm(pool, generator=gen, device=dev)[:total].to(torch.int32)
    width = max(counts)
    rows = torch.repeat_interleave(torch.arange(len(counts), device=dev), torch.tensor(counts, device=dev),
                                   output_size=total)
    first = torch.tensor([sum(counts[:i]) for i in range(len(counts))], device=dev)
    table = torch.full((len(counts), width), -1, dtype=torch.int32, device=dev)
    table[rows, torch.arange(total, device=dev) - first[rows]] = order
    return table, pool


def _cached(gen, case, pool, dev):
    """A cache of whole blocks of keys (a few dimensions far above the others) and values."""
    heads, head, blocks = case["kv_heads"], case["head"], case["page"] // BLOCK
    strong = 1 + 3 * (torch.rand(heads, 1, 1, head, generator=gen, device=dev) < 0.04).float()
    k = torch.empty(pool, heads, case["page"], head, dtype=torch.float8_e4m3fn, device=dev)
    v = torch.empty(pool, heads, blocks, head, BLOCK, dtype=torch.float8_e4m3fn, device=dev)
    k_scales = torch.empty(pool, heads, blocks, device=dev)
    v_scales = torch.empty_like(k_scales)
    step = max(1, (1 << 26) // (heads * case["page"] * head))
    for at in range(0, pool, step):
        count = min(step, pool - at)
        x = torch.randn(count, heads, blocks, BLOCK, head, generator=gen, device=dev) * strong
        s = _powers(x.abs().amax((3, 4)))
        k[at:at + count] = (x / s[..., None, None]).to(torch.float8_e4m3fn).view(count, heads, case["page"], head)
        k_scales[at:at + count] = s
        x = torch.randn(count, heads, blocks, head, BLOCK, generator=gen, device=dev)
        x *= torch.exp(torch.randn(count, heads, blocks, 1, 1, generator=gen, device=dev) * 0.5)
        s = _powers(x.abs().amax((3, 4)))
        v[at:at + count] = (x / s[..., None, None]).to(torch.float8_e4m3fn)
        v_scales[at:at + count] = s
    return k, k_scales, v, v_scales


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dtype = TYPES[case["type"]]
    s = {"op": case["op"]}
    if case["op"] == "adapters":
        rows, k, n = case["requests"] * case["tokens"], case["k"], case["n"]
        x = torch.randn(rows, k, generator=gen, device=dev)
        groups = -(-k // GROUP)
        wide = torch.cat([x, x.new_zeros(rows, groups * GROUP - k)], 1).view(rows, groups, GROUP)
        s["x_scales"] = wide.abs().amax(2) / LARGEST
        s["x"] = (wide / s["x_scales"][:, :, None]).view(rows, -1)[:, :k].contiguous().to(torch.float8_e4m3fn)
        s["down"] = (torch.randn(case["adapters"], case["rank"], k, generator=gen, device=dev) * k ** -0.5).to(dtype)
        s["up"] = (torch.randn(case["adapters"], n, case["rank"], generator=gen, device=dev) * 0.5).to(dtype)
        s["factors"] = 0.5 + torch.rand(case["adapters"], generator=gen, device=dev)
        s["y"] = torch.randn(rows, n, generator=gen, device=dev).to(TYPES[case["result"]])
        request = torch.arange(rows, device=dev) // case["tokens"]
        s["index"] = torch.where(request < case["without"], -1, request % case["adapters"]).to(torch.int32)
        if own:
            from paper_2510_23938_amd import hv
            s["workspace"] = hv.Workspace(dev)
        return s
    new, context = _lengths(case)
    s["new"], s["context"] = new, context  # the program's own counts, beside those on the GPU
    s["starts"] = torch.tensor([sum(new[:i]) for i in range(len(new) + 1)], dtype=torch.int32, device=dev)
    s["lengths"] = torch.tensor(context, dtype=torch.int32, device=dev)
    s["pages"], pool = _pages(gen, case, dev)
    s["cache"] = _cached(gen, case, pool, dev)
    rows = sum(new)
    if case["op"] == "write":
        both = torch.randn(rows, 2, case["kv_heads"], case["head"], generator=gen, device=dev)
        both *= torch.exp(torch.randn(rows, 2, case["kv_heads"], 1, generator=gen, device=dev) * 0.5)
        both = both.to(dtype)
        s["k"], s["v"] = both[:, 0], both[:, 1]
    else:
        s["q"] = torch.randn(rows, case["heads"], case["head"], generator=gen, device=dev).to(dtype)
        s["window"], s["sinks"] = case["window"], case["sinks"]
    if own:
        from paper_2510_23938_amd import hv
        s["cache"] = hv.Fp8Cache(*s["cache"])
        s["workspace"] = hv.Workspace(dev)
    return s


# --------------------------------------------------------------------------
# plain forms

def _plain_write(s):
    k_codes, k_scales, v_codes, v_scales = s["cache"]
    page = k_codes.shape[2]
    dev = k_codes.device
    per_page = page // BLOCK
    # the blocks that new tokens go to: their sequence, and their place in it
    spans = [((c - n) // BLOCK, (c - 1) // BLOCK + 1) for n, c in zip(s["new"], s["context"])]
    total = sum(b - a for a, b in spans)
    counts = torch.tensor([b - a for a, b in spans], device=dev)
    seq = torch.repeat_interleave(torch.arange(len(spans), device=dev), counts, output_size=total)
    before = torch.cumsum(counts, 0) - counts
    lengths, starts = s["lengths"].long(), s["starts"].long()
    first_new = lengths - (starts[1:] - starts[:-1])
    block = torch.arange(total, device=dev) - before[seq] + first_new[seq] // BLOCK
    where = (s["pages"].long()[seq, block // per_page], block % per_page)
    position = block[:, None] * BLOCK + torch.arange(BLOCK, device=dev)
    is_new = (position >= first_new[seq][:, None]) & (position < lengths[seq][:, None])
    is_old = position < first_new[seq][:, None]
    row = (starts[seq][:, None] + position - first_new[seq][:, None]).clamp(0, s["k"].shape[0] - 1)
    for codes, scales, x in ((k_codes.view(k_codes.shape[0], k_codes.shape[1], per_page, BLOCK, -1), k_scales, s["k"]),
                             (v_codes.transpose(3, 4), v_scales, s["v"])):
        x = torch.where(is_new[:, :, None, None], x[row].float(), 0.0).transpose(1, 2)  # [blocks, heads, 16, head]
        finite = torch.where(torch.isfinite(x), x.abs(), 0.0)
        need = _powers(finite.amax((2, 3)))
        held = scales[where[0], :, where[1]]
        scale = torch.where(is_old[:, :1], torch.maximum(need, held), need)
        raw = codes.view(torch.uint8)
        kept_raw = raw[where[0], :, where[1]]
        kept = (kept_raw.view(torch.float8_e4m3fn).float() * (held / scale)[:, :, None, None]).to(torch.float8_e4m3fn)
        fresh = (x / scale[:, :, None, None]).to(torch.float8_e4m3fn)
        out = torch.where(is_new[:, None, :, None], fresh.view(torch.uint8),
                          torch.where(is_old[:, None, :, None], kept.view(torch.uint8), kept_raw))
        raw[where[0], :, where[1]] = out
        scales[where[0], :, where[1]] = scale
    return s["cache"]


def _plain_attention(s):
    k_codes, k_scales, v_codes, v_scales = s["cache"]
    _, kv_heads, page, head = k_codes.shape
    q, out, at = s["q"], [], 0
    heads = q.shape[1]
    dev = q.device
    for i, (n, c) in enumerate(zip(s["new"], s["context"])):
        low = 0 if not s["window"] else max(0, c - n - s["window"] + 1) // page * page
        seen = list(range(0, min(low, -(-s["sinks"] // page) * page), page)) + list(range(low, c, page))
        pages = s["pages"][i, torch.tensor([p // page for p in seen], device=dev)].long()
        token = (torch.tensor(seen, device=dev)[:, None] + torch.arange(page, device=dev)).view(-1)
        k = k_codes[pages].float().view(len(seen), kv_heads, -1, BLOCK, head) * k_scales[pages][..., None, None]
        k = k.permute(1, 0, 2, 3, 4).reshape(kv_heads, -1, head)
        v = v_codes[pages].float() * v_scales[pages][..., None, None]
        v = v.permute(1, 0, 2, 4, 3).reshape(kv_heads, -1, head)
        mine = q[at:at + n].float().view(n, kv_heads, -1, head).transpose(0, 1).reshape(kv_heads, -1, head)
        score = torch.matmul(mine, k.transpose(1, 2)) * head ** -0.5
        place = (c - n + torch.arange(n, device=dev))[:, None]
        allowed = token <= place
        if s["window"]:
            allowed &= (place - token < s["window"]) | (token < s["sinks"])
        score = score.view(kv_heads, n, -1, len(token)).masked_fill(~allowed[None, :, None], -math.inf)
        weight = torch.exp(score - score.amax(3, keepdim=True))
        weight = weight / weight.sum(3, keepdim=True)
        value = torch.matmul(weight.view(kv_heads, -1, len(token)), v * (token < c)[:, None])
        out.append(value.view(kv_heads, n, -1, head).transpose(0, 1).reshape(n, heads, head).to(q.dtype))
        at += n
    return torch.cat(out)


def _plain_adapters(s):
    k, rank = s["x"].shape[1], s["down"].shape[1]
    x = s["x"].float() * s["x_scales"].repeat_interleave(GROUP, 1)[:, :k]
    inner = torch.matmul(x, s["down"].float().view(-1, k).t()).view(x.shape[0], -1, rank)
    mine = s["index"][:, None] == torch.arange(inner.shape[1], device=x.device)
    inner = torch.where(mine[:, :, None], inner * s["factors"][:, None], 0.0).view(x.shape[0], -1)
    up = s["up"].float().transpose(1, 2).reshape(inner.shape[1], -1)
    return (s["y"].float() + torch.matmul(inner, up)).to(s["y"].dtype)


def run(s):
    if not own:
        return {"write": _plain_write, "attention": _plain_attention, "adapters": _plain_adapters}[s["op"]](s)
    from paper_2510_23938_amd import hv
    if s["op"] == "write":
        hv.hv_fp8_cache_write(s["cache"], s["k"], s["v"], s["starts"], s["lengths"], s["pages"])
        return s["cache"].tensors()
    if s["op"] == "attention":
        return hv.hv_fp8_attention(s["q"], s["cache"], s["starts"], s["lengths"], s["pages"], window=s["window"],
                                   sinks=s["sinks"], workspace=s["workspace"])
    return hv.hv_fp8_adapters(s["y"], s["x"], s["x_scales"], s["down"], s["up"], s["index"], s["factors"],
                              workspace=s["workspace"])


# --------------------------------------------------------------------------
# the definitions in 64 bits

def _number_of(codes):
    return codes.float().double()


def exact(case, seed):
    """In the place of 8-bit codes stand the numbers before their rounding, divided by their scale."""
    s = prepare(case, seed)
    if s["op"] == "adapters":
        out = s["y"].double()
        for a in range(s["down"].shape[0]):
            mine = (s["index"] == a).nonzero().view(-1)
            if len(mine) == 0:
                continue
            x = _number_of(s["x"][mine])
            for g in range(s["x_scales"].shape[1]):
                x[:, g * GROUP:(g + 1) * GROUP] *= s["x_scales"][mine, g:g + 1].double()
            out[mine] += s["factors"][a].double() * ((x @ s["down"][a].double().t()) @ s["up"][a].double().t())
        return out
    k_codes, k_scales, v_codes, v_scales = s["cache"].tensors() if own else s["cache"]
    page, head = k_codes.shape[2], k_codes.shape[3]
    table, starts = s["pages"].cpu(), s["starts"].cpu().tolist()
    if s["op"] == "write":
        if k_codes.numel() > 1 << 28 or sum(s["new"]) > 40000:
            return None
        k_out, v_out = _number_of(k_codes), _number_of(v_codes)
        k_s, v_s = k_scales.clone(), v_scales.clone()
        for i, (n, c) in enumerate(zip(s["new"], s["context"])):
            for b in range((c - n) // BLOCK, (c - 1) // BLOCK + 1):
                low, high = max(c - n, b * BLOCK), min(c, (b + 1) * BLOCK)
                rows = slice(starts[i] + low - (c - n), starts[i] + high - (c - n))
                a, z = low - b * BLOCK, high - b * BLOCK
                p, in_page = int(table[i, b * BLOCK // page]), b % (page // BLOCK)
                at = in_page * BLOCK
                for x, codes, scales in ((s["k"], k_out[p, :, at:at + BLOCK], k_s),
                                         (s["v"], v_out[p, :, in_page].transpose(1, 2), v_s)):
                    x = x[rows].double().transpose(0, 1)
                    top = x.abs().amax((1, 2))
                    need = torch.exp2(torch.ceil(torch.log2(top / LARGEST)).clamp_min(-126))
                    held = scales[p, :, in_page].double()
                    scale = torch.maximum(need, held) if a > 0 else need
                    codes[:, :a] *= (held / scale)[:, None, None]
                    codes[:, a:z] = x / scale[:, None, None]
                    scales[p, :, in_page] = scale.float()
        return k_out, k_s, v_out, v_s
    q = s["q"]
    out = torch.empty(q.shape, dtype=torch.float64, device=q.device)
    share = q.shape[1] // k_codes.shape[1]
    for i, (n, c) in enumerate(zip(s["new"], s["context"])):
        token = torch.arange(c, device=q.device)
        own_pages = s["pages"][i, token // page].long()
        slot = token % page
        place = torch.arange(c - n, c, device=q.device)
        hidden = token[None, :] > place[:, None]
        if s["window"]:
            hidden |= (token[None, :] <= place[:, None] - s["window"]) & (token[None, :] >= s["sinks"])
        for h in range(k_codes.shape[1]):
            keys = _number_of(k_codes[own_pages, h, slot]) * k_scales[own_pages, h, slot // BLOCK].double()[:, None]
            values = _number_of(v_codes[own_pages, h, slot // BLOCK, :, slot % BLOCK])
            values = values * v_scales[own_pages, h, slot // BLOCK].double()[:, None]
            for g in range(share):
                rows = q[starts[i]:starts[i + 1], h * share + g].double()
                score = (rows @ keys.t().contiguous()) / math.sqrt(head)
                score[hidden] = -math.inf
                out[starts[i]:starts[i + 1], h * share + g] = torch.softmax(score, 1) @ values
    return out
