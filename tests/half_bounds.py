"""What attention in half precision over the 8-bit cache may differ by from its value in 64 bits, row by row.

As in cache_bounds.py, but for weights that are subnormal numbers of the type.  A weight w, relative to its row's largest,
is rounded as p = w * 2^(e - most + 4), with e the exponent of its block's value scale and `most` the largest of those that the row
sees.  (The row's maximum may lag by L of up to 2^8, and p be that much larger: what is lost divided by L is no more.)  Below
2^-14 that loses up to 2^-25, or all of p if that is less; its code's product with it, by 2^(most - 4) and divided by the weights'
sum, is what the output loses.  The result loses up to 2^-25 where it is subnormal."""
import numpy as np

from oracle import fp8, fp8_cache

HALF = 2.0 ** -11


def subnormal_losses(cache, q, starts, lengths, table, scale):
    """[tokens, heads, dim], without windows."""
    tokens, heads, dim = q.shape
    lost = np.zeros(q.shape)
    share = heads // cache.heads
    for i, rows, position in fp8_cache.sequences(starts, lengths, tokens):
        spots = [(j, fp8_cache.place(cache, table, i, j)) for j in range(position + len(rows))]
        at = np.array([j for j, p in spots if p is not None])
        page, block, slot = np.array([p for _, p in spots if p is not None]).T
        for g in range(cache.heads):
            keys = fp8.VALUES[cache.k[page, g, block * 16 + slot]] * cache.ks[page, g, block].astype(np.float64)[:, None]
            codes = np.abs(fp8.VALUES[cache.v[page, g, block, :, slot]])
            e = np.log2(cache.vs[page, g, block].astype(np.float64))
            for h in range(g * share, (g + 1) * share):
                for n, row in enumerate(rows):
                    seen = at <= position + n
                    s = keys[seen] @ q[row, h] * scale
                    w = np.exp(s - s.max())
                    p = w * 2.0 ** (e[seen] - e[seen].max() + 4)
                    small = p < 2.0 ** -14
                    lost[row, h] = np.minimum(p, 2.0 ** -25)[small] @ codes[seen][small] * 2.0 ** (e[seen].max() - 4) / w.sum()
    return lost


def check(got, want, lost):
    out, size, root, steep = want
    weights = 2 * (100 * 2.0 ** -24 * steep + 2.0 ** -21 + 2.0 ** -18)[:, :, None]
    allowed = weights * size + 6 * HALF / np.sqrt(3) * root + HALF * np.abs(out) + lost + 2.0 ** -25
    off = np.abs(got - out)
    assert (off <= allowed).all(), (np.argwhere(~(off <= allowed))[:5], np.nanmax(off / allowed))
