"""The 8-bit cache and the attention over it from their definitions, in 64 bits on the host (numpy).

Codes are uint8 arrays.  Shares no code with the HIP path.
"""
import math

import numpy as np

from oracle.fp8 import LARGEST, VALUES, round_to_code

BLOCK = 16


def power_scale(largest: float) -> float:
    """The smallest power of two, at least 2^-126, under which this is at most 448."""
    scale = 2.0 ** -126
    while largest > LARGEST * scale:
        scale *= 2
    return scale


class Cache:
    """k [pages, heads, tokens, dim], v [pages, heads, tokens / 16, dim, 16]: codes; ks, vs [pages, heads, tokens / 16]."""

    def __init__(self, k, ks, v, vs):
        self.k, self.ks, self.v, self.vs = (np.array(a) for a in (k, ks, v, vs))
        self.pages, self.heads, self.page_tokens, self.dim = self.k.shape

    def copy(self):
        return Cache(self.k, self.ks, self.v, self.vs)

    def keys(self, page, head, block):
        """Codes of a block's keys, [16, dim], as a view."""
        return self.k[page, head, block * BLOCK:(block + 1) * BLOCK]

    def values(self, page, head, block):
        return self.v[page, head, block].T


def sequences(starts, lengths, tokens):
    """(sequence, its rows, the position of the first) of those that a batch describes."""
    for i in range(len(lengths)):
        first, end = int(starts[i]), int(starts[i + 1])
        if 0 <= first < end <= tokens:
            yield i, range(first, end), max(int(lengths[i]), 0) - (end - first)


def place(cache, table, i, position):
    """(page, block in it, slot in that) of a position, or None where the cache has none."""
    if not 0 <= position < table.shape[1] * cache.page_tokens:
        return None
    page = int(table[i, position // cache.page_tokens])
    if not 0 <= page < cache.pages:
        return None
    return page, position % cache.page_tokens // BLOCK, position % BLOCK


def write(cache, k, v, starts, lengths, table):
    """Writes rows of k and v [tokens, heads, dim] (64 bits) to the cache, in place."""
    for i, rows, position in sequences(starts, lengths, len(k)):
        blocks = {}
        for n, row in enumerate(rows):
            at = place(cache, table, i, position + n)
            if at is not None:
                blocks.setdefault(at[:2], []).append((at[2], row))
        for (page, block), new in blocks.items():
            for head in range(cache.heads):
                for x, codes, scales in ((k, cache.keys(page, head, block), cache.ks),
                                         (v, cache.values(page, head, block), cache.vs)):
                    y = np.stack([x[row, head] for _, row in new]).astype(np.float64)
                    a = np.abs(y)
                    scale = power_scale(a[np.isfinite(a)].max(initial=0.0))
                    first = new[0][0]
                    if first > 0:
                        held = float(scales[page, head, block])
                        scale = max(scale, held)
                        if scale != held:
                            codes[:first] = round_to_code(VALUES[codes[:first]] * (held / scale))
                    for (slot, _), row in zip(new, y):
                        codes[slot] = round_to_code(row / scale)
                    scales[page, head, block] = scale


def attention(cache, q, starts, lengths, table, scale, window=0, sinks=0):
    """Attention of q [tokens, heads, dim] (64 bits), (out, size, root, steep): the outputs, and what bounds their
    rounding: size = sum of w |v|, root = the root of the sum of (w v)^2, and steep [tokens, heads], the largest sum of
    |q k| * scale of a visible key.  Rows of no sequence are NaN."""
    tokens, heads, dim = q.shape
    out, size, root = (np.full(q.shape, np.nan) for _ in range(3))
    steep = np.zeros((tokens, heads))
    share = heads // cache.heads
    for i, rows, position in sequences(starts, lengths, tokens):
        spots = [(j, place(cache, table, i, j)) for j in range(max(position + len(rows), 0))]
        spots = [(j, p) for j, p in spots if p is not None]
        at = np.array([j for j, _ in spots], dtype=np.int64)
        page, block, slot = np.array([p for _, p in spots], dtype=np.int64).reshape(-1, 3).T
        pos = position + np.arange(len(rows))[:, None]
        seen = at[None, :] <= pos
        if window:
            seen &= (pos - at[None, :] < window) | (at[None, :] < sinks)
        for head in range(cache.heads):
            keys = VALUES[cache.k[page, head, block * BLOCK + slot]] * cache.ks[page, head, block].astype(np.float64)[:, None]
            vals = VALUES[cache.v[page, head, block, :, slot]] * cache.vs[page, head, block].astype(np.float64)[:, None]
            for h in range(head * share, (head + 1) * share):
                for n, row in enumerate(rows):
                    vis = seen[n]
                    if not vis.any():
                        out[row, h] = size[row, h] = root[row, h] = 0.0
                        continue
                    k, v = keys[vis], vals[vis]
                    s = (k @ q[row, h]) * scale
                    w = np.exp(s - s.max()) if np.isfinite(s).all() else np.full(s.shape, math.nan)
                    w /= w.sum()
                    out[row, h], size[row, h] = w @ v, w @ np.abs(v)
                    root[row, h] = np.sqrt((w * w) @ (v * v))
                    steep[row, h] = (np.abs(k) @ np.abs(q[row, h])).max() * scale
    return out, size, root, steep
