"""The attention half of a decoder layer in 64 bits, from its definition: the documented places of the paged cache, rotary positions,
causal attention.  Plain numpy on the host; shares nothing with the library."""
import numpy as np

BF16_HALF_STEP = 2.0 ** -8          # a rounding to bf16, relative to the value
F32_HALF_STEP = 2.0 ** -24


def padded(D):
    return (D + 7) // 8 * 8


def bf16(x):
    """fp64 -> the nearest bf16 (ties to even), as fp64, through fp32 bits; for inputs that are fp32 already."""
    u = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    u = (u + 0x7FFF + ((u >> 16) & 1)) & 0xFFFF0000
    return u.astype(np.uint32).view(np.float32).astype(np.float64)


class Cache:
    """Pages on the host, [pages][tokens][heads][D] in the natural order, with the conversions to and from the documented layout."""

    def __init__(self, pages, page_tokens, kv_heads, D, fill=np.nan):
        self.pages, self.P, self.H, self.D = pages, page_tokens, kv_heads, D
        self.k = np.full((pages, page_tokens, kv_heads, D), fill, dtype=np.float32)
        self.v = np.full((pages, page_tokens, kv_heads, D), fill, dtype=np.float32)

    def put(self, row, first, k, v):
        """k, v [n, heads, D] at positions first ... of the sequence with the table row `row`."""
        for i in range(len(k)):
            page, at = row[(first + i) // self.P], (first + i) % self.P
            if 0 <= page < self.pages:
                self.k[page, at], self.v[page, at] = k[i], v[i]

    def get(self, row, n):
        """(keys, values, whether there is such a page) of positions 0 ... n - 1, fp64."""
        pos = np.arange(n)
        page = np.asarray(row)[pos // self.P]
        there = (page >= 0) & (page < self.pages)
        page = np.where(there, page, 0)
        return self.k[page, pos % self.P].astype(np.float64), self.v[page, pos % self.P].astype(np.float64), there

    def layout(self):
        """fp32 arrays in the documented order (to be cast to bf16): keys [pages, heads, blocks, Dp / 8, 32, 8], values [..., 4, Dp, 8]."""
        Dp, nb = padded(self.D), self.P // 32
        k = np.zeros((self.pages, self.H, nb, Dp // 8, 32, 8), dtype=np.float32)
        v = np.zeros((self.pages, self.H, nb, 4, Dp, 8), dtype=np.float32)
        t, d = np.arange(self.P)[:, None], np.arange(self.D)[None, :]
        j = t % 32
        k[:, :, t // 32, d // 8, 16 * ((j >> 2) & 1) + 4 * (j >> 3) + (j & 3), d % 8] = self.k.transpose(0, 2, 1, 3)
        v[:, :, t // 32, j >> 3, d, j & 7] = self.v.transpose(0, 2, 1, 3)
        return k, v

    def from_layout(self, k, v):
        """(keys, values) in the natural order out of arrays in the documented one."""
        t, d = np.arange(self.P)[:, None], np.arange(self.D)[None, :]
        j = t % 32
        return (k[:, :, t // 32, d // 8, 16 * ((j >> 2) & 1) + 4 * (j >> 3) + (j & 3), d % 8].transpose(0, 2, 1, 3),
                v[:, :, t // 32, j >> 3, d, j & 7].transpose(0, 2, 1, 3))


def rope(x, pos, freq, pairs):
    """x [n, heads, D] fp64 at positions pos [n] -> (turned, bound of the fp32 steps): the angle in 64 bits, then at most 2^-21 on sine and
    cosine (a fraction of a turn rounded to fp32, pi times it, the function itself) and three fp32 roundings."""
    y, r = x.copy(), 2 * len(freq)
    half = len(freq)
    a = (slice(0, r, 2), slice(1, r, 2)) if pairs else (slice(0, half), slice(half, r))
    angle = pos.astype(np.float64)[:, None, None] * freq.astype(np.float64)
    c, s = np.cos(angle), np.sin(angle)
    p, q = x[..., a[0]], x[..., a[1]]
    y[..., a[0]], y[..., a[1]] = p * c - q * s, q * c + p * s
    off = np.zeros_like(x)
    off[..., a[0]] = off[..., a[1]] = (np.abs(p) + np.abs(q)) * (2.0 ** -21 + 3 * F32_HALF_STEP)
    return y, off


def attention(q, k, v, seen, scale):
    """q [heads, D] of one row over k, v [n, kv heads, D]; seen [n] -> (o [heads, D], (the bounds of a bf16 and an fp32 result)).

    The bounds: scores in fp32 are off by at most (D + 8) half steps of sum |q k| (times scale, in the exponent; the steps of exp2 and of
    the running maximum are in the 8), so a weight by that relative error; sums over the keys by a half step for each of their terms, once
    over the values and once over the weights.  Weights are rounded to bf16 (half a step each), or to the sum of two bf16 (half a
    step of half a step); the result is rounded once."""
    heads, D = q.shape
    kv_heads = k.shape[1]
    o, bb, fb = np.zeros((heads, D)), np.zeros((heads, D)), np.zeros((heads, D))
    if not seen.any():
        return o, (bb, fb)
    for h in range(heads):
        kh, vh = k[seen, h * kv_heads // heads], v[seen, h * kv_heads // heads]
        s = kh @ q[h] * scale
        p = np.exp(s - s.max())
        p /= p.sum()
        o[h] = p @ vh
        size = p @ np.abs(vh)
        by = 2 * (D + 8) * F32_HALF_STEP * scale * (np.abs(kh) @ np.abs(q[h])).max() + (2 * len(kh) + 64) * F32_HALF_STEP
        fb[h] = size * (by + BF16_HALF_STEP ** 2) * 1.01 + F32_HALF_STEP * np.abs(o[h]) + 1e-37
        bb[h] = size * (by + BF16_HALF_STEP) * 1.01 + BF16_HALF_STEP * 1.01 * np.abs(o[h]) + 1e-37
    return o, (bb, fb)
