"""What a serving loop does around the paged cache in 64 bits, from its definition: normed heads, weights of cached tokens, eviction.  Plain numpy on the
host; shares nothing with the library."""
import numpy as np

from attention_ref import F32_HALF_STEP, rope


def norm_rope(x, pos, freq, pairs, gain, eps, norm):
    """x [n, heads, D] fp64 -> (normed and turned, bound of the fp32 steps).  A head's sum of squares is one of positive terms in fp32: up to 16 steps of a
    lane and 5 between lanes, a half step of the sum each, so 21, of which the root takes half; the mean's product and the sum with eps one each, of
    which the root takes half; the root's instruction two: 13.5 half steps on the factor.  Its two products have one each, and go
    through the turn with both of a pair."""
    if not norm:
        return rope(x, pos, freq, pairs)
    s = (x * x).mean(axis=-1, keepdims=True)
    y = np.where(s > 0, x / np.sqrt(np.where(s > 0, s + eps, 1.0)), 0.0) * (1.0 if gain is None else gain.astype(np.float64))
    z, off = rope(y, pos, freq, pairs)
    r, half = 2 * len(freq), len(freq)
    size = np.abs(y)
    a = (slice(0, r, 2), slice(1, r, 2)) if pairs else (slice(0, half), slice(half, r))
    size[..., a[0]] = size[..., a[1]] = size[..., a[0]] + size[..., a[1]]
    return z, off + 15.5 * F32_HALF_STEP * size


def weights(q, k, seen, scale):
    """q [heads, D] of one row over k [n, kv heads, D]; seen [n] -> (softmax weights summed over the heads of each key-value head [kv heads, n], their
    bounds).  Scores in fp32 are off by at most (D + 8) half steps of sum |q k| (in the exponent, with the steps of exp2 and the running maximum in the
    8), so is the sum that divides them, which has a half step for each of its terms too; the sum over the heads has one for each."""
    heads, D = q.shape
    kv_heads, n = k.shape[1], len(seen)
    w, off = np.zeros((kv_heads, n)), np.zeros((kv_heads, n))
    if not seen.any():
        return w, off
    for h in range(heads):
        g = h * kv_heads // heads
        kh = k[seen, g]
        s = kh @ q[h] * scale
        p = np.exp(s - s.max())
        p /= p.sum()
        by = 2 * (D + 8) * F32_HALF_STEP * scale * (np.abs(kh) @ np.abs(q[h])).max() + (n + 64) * F32_HALF_STEP
        w[g, seen] += p
        off[g, seen] += p * (by + heads // kv_heads * F32_HALF_STEP)
    return w, off * 1.01 + 1e-38


def evict(w, n, keep, recent):
    """The positions that stay of one head's n tokens with the weights w: the `recent` last, and the heaviest others, of equal ones the lower, in order."""
    late = 0 if n <= keep else n - recent
    order = sorted(range(late), key=lambda p: (-(np.inf if np.isnan(w[p]) else w[p]), not np.isnan(w[p]), p))
    return sorted(order[: keep - (n - late)]) + list(range(late, n))
