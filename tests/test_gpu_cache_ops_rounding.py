"""How often the results of the cache's attention operators are rounded: a bf16 result once, however many sequences share a prefix and however long a run is."""
import numpy as np
import pytest

from attention_ref import BF16_HALF_STEP, attention
from test_gpu_attention import Batch, dev, dev16, host
from test_gpu_cache_ops import Shared

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

DIMS = [2, 24, 64, 100, 128, 160, 256]


def rounded_once(got, q, k, v, seen, label):
    """Weights of two bf16 operands leave 2^-17 of each, in the sums over the values, which the bound of attention_ref for fp32 results (2^-16, its scores and
    sums) has room for; the result's own half step comes on top and nothing of a weight's half step."""
    heads, D = q.shape
    o, (_, once) = attention(q, np.where(seen[:, None, None], k, 0), np.where(seen[:, None, None], v, 0), seen, D ** -0.5)
    off, most = np.abs(got.reshape(heads, D) - o), once + BF16_HALF_STEP * (np.abs(o) + once)
    assert (off <= most).all(), (label, (off / most).max())


# 6, 192 and 320 rows a key-value head: one launch for shared and own tokens; two launches; tiles of 128 rows where heads have up to 128 dims
@pytest.mark.parametrize("lens,counts,prefixes,heads,kv_heads", [
    ([700, 641, 600, 900, 5, 1300], [4, 2], [640, 3], 2, 2), ([700 + 3 * (b % 7) for b in range(24)], [24], [650], 16, 2),
    ([700 + 90 * (b % 7) - 600 * (b % 13 == 12) for b in range(40)], [40], [650], 16, 2)])
@pytest.mark.parametrize("D", DIMS)
def test_shared_prefixes(gpu_lib, lens, counts, prefixes, heads, kv_heads, D):
    batch = Shared(lens, counts, prefixes, 32, kv_heads, D, 91)
    q = batch.queries(len(lens), heads, D)
    y = host(gpu_lib.attention_decode_shared(dev16(q), batch.k, batch.v, dev(batch.table), dev(lens), dev(batch.start), dev(batch.prefix), y_dtype=gpu_lib.BF16))
    for b in range(0, len(lens), 1 if len(lens) < 10 else 5):
        rounded_once(y[b], q[b], *batch.keys_of(b), b)


# one launch; rows that workgroups share
@pytest.mark.parametrize("lens", [[1, 2, 31, 33, 64, 0, 127, 129, 300], [5000], [4097, 1, 2050]])
@pytest.mark.parametrize("D", DIMS)
def test_decode_weights(gpu_lib, lens, D):
    heads, kv_heads = 6, 2
    batch = Batch(lens, 96, kv_heads, D, 92)
    q, acc = batch.queries(len(lens), heads, D), torch.zeros((len(lens), kv_heads, batch.per * 96), device="cuda")
    y = host(gpu_lib.attention_decode_weights(dev16(q), batch.k, batch.v, dev(batch.table), dev(lens), acc, y_dtype=gpu_lib.BF16))
    for b, n in enumerate(lens):
        rounded_once(y[b], q[b], *batch.cache.get(batch.table[b], n), n)


# tiles of 64 rows; rows that workgroups share; tiles of 128 rows, of a chunk behind others and of a prompt in a table that has room for more
@pytest.mark.parametrize("sizes,heads,kv_heads,per", [([(0, 300), (45, 1), (130, 70)], 4, 2, None), ([(3000, 5)], 4, 2, None), ([(4500, 1030)], 64, 8, None), ([(0, 300)], 256, 32, 20)])
@pytest.mark.parametrize("D", DIMS)
def test_prefill_weights(gpu_lib, sizes, heads, kv_heads, per, D):
    lens, starts = [o + n for o, n in sizes], np.cumsum([0] + [n for _, n in sizes])
    batch = Batch(lens, 64, kv_heads, D, 93, per)
    T = int(starts[-1])
    q, acc = batch.queries(T, heads, D), torch.zeros((len(lens), kv_heads, batch.per * 64), device="cuda")
    y = host(gpu_lib.attention_prefill_weights(dev16(q), batch.k, batch.v, dev(batch.table), dev(lens), dev(starts), acc, y_dtype=gpu_lib.BF16))
    for b, (old, n) in enumerate(sizes):
        k, v, there = batch.cache.get(batch.table[b], lens[b])
        for i in sorted({0, n - 1} | set(int(i) for i in batch.rng.integers(0, n, 5))):
            rounded_once(y[starts[b] + i], q[starts[b] + i], k, v, there & (np.arange(lens[b]) <= old + i), (b, i))
