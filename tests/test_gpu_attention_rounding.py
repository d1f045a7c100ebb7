"""How often attention's results are rounded: the divisor of a softmax takes the weights as the values' product does."""
import numpy as np
import pytest

from attention_ref import BF16_HALF_STEP, attention
from test_gpu_attention import Batch, dev, dev16, host

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


# the last two: rows that workgroups share, and tiles of 128 rows
@pytest.mark.parametrize("sizes,heads,kv_heads", [([(0, 300), (45, 1), (130, 70)], 4, 2), ([(3000, 5)], 4, 2), ([(4500, 1030)], 64, 8)])
@pytest.mark.parametrize("D", [24, 64, 100, 128, 160, 256])
@pytest.mark.parametrize("f32", [False, True])
def test_values_all_alike_come_back(gpu_lib, sizes, heads, kv_heads, D, f32):
    """sum(w c) / sum(w) is c, a bf16, whatever the weights are: the sums go over n terms in 32 bits, so their quotient is within
    (2 n + 64) 2^-24 of c, which for n < 10000 is less than the 2^-9 from which on a bf16 would be another one.  Scores of a
    standard deviation of 3 to 5: a few weights count, and the roundings of many do not cancel."""
    n = sum(o + t for o, t in sizes)
    batch = Batch([o + t for o, t in sizes], 64, kv_heads, D, 31)
    alike = dev16(batch.rng.uniform(0.5, 2.0, (kv_heads, D)))
    c = host(alike)
    batch.cache.v[:] = np.where(np.isnan(batch.cache.v), np.nan, c.astype(np.float32))
    v = dev16(batch.cache.layout()[1])
    T = sum(t for _, t in sizes)
    q = dev16(batch.queries(T, heads, D, 4.0))
    kind = gpu_lib.F32 if f32 else gpu_lib.BF16
    lens = dev(batch.lens)
    y = gpu_lib.attention_prefill(q, batch.k, v, dev(batch.table), lens, dev(np.cumsum([0] + [t for _, t in sizes])), y_dtype=kind)
    last = np.cumsum([t for _, t in sizes]) - 1
    one = gpu_lib.attention_decode(q[dev(last, np.int64)], batch.k, v, dev(batch.table), lens, y_dtype=kind)
    for got in (y, one):
        off = np.abs(host(got).reshape(-1, kv_heads, heads // kv_heads, D) / c[:, None, :] - 1)
        assert off.max() <= ((2 * n + 64) * 2.0 ** -24 if f32 else 0.0), off.max()


# one launch (up to three rounds of blocks, a sequence of no tokens), rows that workgroups share
@pytest.mark.parametrize("lens", [[1, 2, 31, 33, 64, 0, 127, 129, 300], [5000], [4097, 1, 2050]])
@pytest.mark.parametrize("D", [2, 24, 64, 100, 128, 160, 256])
def test_decode_rounds_a_bf16_result_once(gpu_lib, lens, D):
    """Weights of two bf16 operands leave 2^-17 of each, in the sums and in the divisor, which the bound of attention_ref for fp32 results
    (2^-16, its scores and sums) has room for; the result's own half step comes on top and nothing of a weight's half step."""
    heads, kv_heads = 6, 2
    batch = Batch(lens, 96, kv_heads, D, 32)
    q = batch.queries(len(lens), heads, D)
    y = host(gpu_lib.attention_decode(dev16(q), batch.k, batch.v, dev(batch.table), dev(lens), y_dtype=gpu_lib.BF16))
    for b, n in enumerate(lens):
        k, v, there = batch.cache.get(batch.table[b], n)
        o, (_, once) = attention(q[b], k, v, there, D ** -0.5)
        off = np.abs(y[b].reshape(heads, D) - o)
        assert (off <= once + BF16_HALF_STEP * (np.abs(o) + once)).all(), (n, (off / (once + BF16_HALF_STEP * np.abs(o))).max())
