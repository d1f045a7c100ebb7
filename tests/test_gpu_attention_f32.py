"""fp32 results of attention keep their weights whole: scores that are exact, two keys that count, and a bound that weights of two bf16
operands (16 bits) fail.

q has 16 and a (1 ... 127) in its first two dims.  The keys are zeros at one place, (0, -1) at another, (-2^14, 0) at all others: scores of 0,
-a and -2^18, times 2^-7, so the weights are 1, p = exp(-a / 128) and zeros, in steps of
  exponents: fl(score scale log2 e - base), base = fl(maximum scale log2 e), the constant: 1.44 + 1.44 + 0.72 half steps, times ln 2, and a
    unit in the last place of exp2: 4.5 half steps for a weight, 9 for a quotient of two; as many for the factors with which waves
    or workgroups join: 18 half steps e.  With values +-1 the result moves by 2 p e / (1 + p)^2 <= e / 2;
  sums: at most five additions of six products that are exact, and a factor for each move of the maximum, join of waves, join of
    workgroups: 10 half steps of sum(w |v|), 10 of sum(w), two of the quotient.
"""
import numpy as np
import pytest

from attention_ref import F32_HALF_STEP, bf16
from test_gpu_attention import Batch, dev, dev16, host

torch = pytest.importorskip("torch")

SCALE, FAR = 2.0 ** -7, -2.0 ** 14


def exact(a, v0, v1):
    """a [rows, heads], v0, v1 [heads, D] (the values of the two keys that count) -> (o [rows, heads, D], its bound)."""
    p = np.exp(-a * SCALE)[..., None]
    o = (v0 + p * v1) / (1 + p)
    size = (np.abs(v0) + p * np.abs(v1)) / (1 + p)
    return o, F32_HALF_STEP * (18 * p / (1 + p) ** 2 * np.abs(v0 - v1) + 10 * size + 12 * np.abs(o))


def counts(rows, heads):
    return 1.0 + np.arange(rows * heads).reshape(rows, heads) % 127


def values(rng, heads, D):
    """of the two keys: about 1 and about -1."""
    return bf16(rng.uniform(0.75, 1.0, (heads, D))), -bf16(rng.uniform(0.75, 1.0, (heads, D)))


@pytest.mark.parametrize("parts,passes", [(1, False), (2, False), (3, True)])
def test_the_bound_tells_the_number_of_operands(parts, passes):
    """Weights of one, two and three bf16 in the definition itself: the first two are out of bounds, whether the divisor takes them so or whole."""
    a = counts(127, 1)
    v0, v1 = values(np.random.default_rng(1), 1, 64)
    o, bound = exact(a, v0, v1)
    p = np.exp(-a * SCALE).astype(np.float32).astype(np.float64)
    kept, rest = np.zeros_like(p), p
    for _ in range(parts):
        kept, rest = kept + bf16(rest), rest - bf16(rest)
    for divisor in (kept, p):
        off = np.abs((v0 + kept[..., None] * v1) / (1 + divisor[..., None]) - o)
        assert (off <= bound).all() == passes


def batch_of(lens, places, kv_heads, D):
    batch = Batch(lens, 64, kv_heads, D, 41)
    c, v = batch.cache, values(batch.rng, kv_heads, D)
    held = ~np.isnan(c.k[..., 0])
    c.k[held] = np.concatenate([[FAR], np.zeros(D - 1)])
    for b, (first, second) in enumerate(places):
        for at, key, value in ((first, 0, v[0]), (second, -1, v[1])):
            page = batch.table[b, at // c.P]
            c.k[page, at % c.P] = np.concatenate([[0, key], np.zeros(D - 2)])
            c.v[page, at % c.P] = value
    k, w = c.layout()
    batch.k, batch.v = dev16(k), dev16(w)
    return batch, v


def queries(a, D):
    q = np.zeros(a.shape + (D,))
    q[..., 0], q[..., 1] = 16, a
    return dev16(q)


def check(y, a, v, kv_heads, D):
    rows, heads = a.shape
    o, bound = exact(a, *(np.repeat(x, heads // kv_heads, axis=0) for x in v))
    off = np.abs(host(y).reshape(rows, heads, D) - o)
    assert (off <= bound).all(), (off / bound).max()


DIMS = [24, 32, 64, 100, 128, 160, 192, 256]


# one launch; rows that workgroups share, with both keys in one's part and in two
@pytest.mark.gpu
@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("lens,places", [([300] * 32, [(b, 299 - 3 * b) for b in range(32)]), ([5000, 4000], [(10, 4000), (3999, 3990)])])
def test_decode(gpu_lib, D, lens, places):
    batch, v = batch_of(lens, places, 2, D)
    a = counts(len(lens), 64)
    y = gpu_lib.attention_decode(queries(a, D), batch.k, batch.v, dev(batch.table), dev(lens), SCALE, gpu_lib.F32)
    check(y, a, v, 2, D)


# tiles of 64 rows, rows that workgroups share, tiles of 128 rows
@pytest.mark.gpu
@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("old,new,heads,kv_heads,place", [(300, 70, 4, 2, (290, 5)), (3000, 16, 8, 2, (10, 2900)), (4500, 1030, 64, 8, (4400, 70))])
def test_prefill(gpu_lib, D, old, new, heads, kv_heads, place):
    batch, v = batch_of([old + new], [place], kv_heads, D)
    a = counts(new, heads)
    y = gpu_lib.attention_prefill(queries(a, D), batch.k, batch.v, dev(batch.table), dev([old + new]), dev([0, new]), SCALE, gpu_lib.F32)
    check(y, a, v, kv_heads, D)
