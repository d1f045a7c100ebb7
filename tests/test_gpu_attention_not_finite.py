"""Values that are not finite: a row that sees one has NaN in its dim of the heads that read it, whichever kernel, tile or workgroup takes the
row, and all else is what it is without it."""
import numpy as np
import pytest

from test_gpu_attention import Batch, dev, dev16, host

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

INF, NAN = np.inf, np.nan


def caches(D, old, new, kv_heads, marks):
    """marks: {position: value} in dim 1 of key-value head 0 -> (batch, its values, its values with the marks)."""
    batch = Batch([old + new], 32, kv_heads, D, 51)
    plain = batch.v
    for at, value in marks.items():
        batch.cache.v[batch.table[0, at // 32], at % 32, 0, 1] = value
    return batch, plain, dev16(batch.cache.layout()[1])


def check(got, want, heads, kv_heads, D, positions, first):
    got, want = host(got).reshape(-1, heads, D), host(want).reshape(-1, heads, D)
    touched = np.zeros(got.shape, dtype=bool)
    touched[np.asarray(positions) >= first, : heads // kv_heads, 1] = True
    assert np.isnan(got[touched]).all() and np.array_equal(got[~touched], want[~touched])


# in stages that all rows of a tile see and in those that some do not, next to a page's end, several and of both signs;
# rows that workgroups share, tiles of 128 rows
@pytest.mark.parametrize("old,new,heads,kv_heads,marks", [
    (0, 300, 4, 2, {40: INF}), (0, 300, 4, 2, {299: -INF}), (0, 300, 4, 2, {0: NAN}), (33, 130, 6, 2, {5: -INF, 64: INF}), (33, 130, 6, 2, {63: INF, 64: INF}),
    (0, 1, 4, 2, {0: INF}), (3000, 5, 4, 2, {2999: INF}), (3000, 5, 4, 2, {7: -INF}), (3000, 5, 4, 2, {3002: INF}), (3200, 1030, 64, 8, {9: INF}), (3200, 1030, 64, 8, {3600: -INF})])
@pytest.mark.parametrize("D", [24, 64, 100, 128, 192])
@pytest.mark.parametrize("f32", [False, True])
def test_prefill(gpu_lib, old, new, heads, kv_heads, marks, D, f32):
    batch, plain, v = caches(D, old, new, kv_heads, marks)
    q = dev16(batch.queries(new, heads, D))
    y, want = (gpu_lib.attention_prefill(q, batch.k, x, dev(batch.table), dev([old + new]), dev([0, new]), y_dtype=gpu_lib.F32 if f32 else gpu_lib.BF16) for x in (v, plain))
    check(y, want, heads, kv_heads, D, np.arange(old, old + new), min(marks))


@pytest.mark.parametrize("n,at", [(1, 0), (77, 3), (77, 76), (300, 150), (5000, 1), (5000, 4999)])
@pytest.mark.parametrize("value", [INF, -INF, NAN])
@pytest.mark.parametrize("D", [24, 64, 100, 128, 192])
@pytest.mark.parametrize("f32", [False, True])
def test_decode(gpu_lib, n, at, value, D, f32):
    batch, plain, v = caches(D, n - 1, 1, 2, {at: value})
    q = dev16(batch.queries(1, 8, D))
    y, want = (gpu_lib.attention_decode(q, batch.k, x, dev(batch.table), dev([n]), y_dtype=gpu_lib.F32 if f32 else gpu_lib.BF16) for x in (v, plain))
    check(y, want, 8, 2, D, [n - 1], at)
