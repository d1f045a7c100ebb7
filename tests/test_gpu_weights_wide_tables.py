"""Weights of cached tokens in runs, where page tables have room for more than their sequences: how the work is shared out goes by the sequences."""
import numpy as np
import pytest

from test_gpu_attention import Batch, dev, dev16
from test_gpu_cache_ops import run_weights

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def weighed(gpu_lib, batch, per, sizes, heads, D, f32, seed):
    """The accumulators of a call whose table rows are `per` pages long, and the attention."""
    table = np.full((len(sizes), per), -1, dtype=np.int32)
    table[:, : batch.per] = batch.table
    lens, starts = [o + n for o, n in sizes], np.cumsum([0] + [n for _, n in sizes])
    q = dev16(np.random.default_rng(seed).standard_normal((int(starts[-1]), heads, D)))
    acc = torch.zeros((len(sizes), batch.cache.H, per * batch.cache.P), device="cuda")
    y = gpu_lib.attention_prefill_weights(q, batch.k, batch.v, dev(table), dev(lens), dev(starts), acc, y_dtype=gpu_lib.F32 if f32 else gpu_lib.BF16)
    return y, acc[:, :, : batch.per * batch.cache.P].contiguous()


# the attention in front takes one launch, whatever room there is: its rows fill the chip
@pytest.mark.parametrize("sizes,heads,kv_heads", [([(0, 300)] * 4, 32, 32), ([(0, 500), (0, 31), (0, 257), (0, 480)], 32, 32), ([(0, 1000)], 64, 8)])
@pytest.mark.parametrize("D", [64, 100, 128, 160])
@pytest.mark.parametrize("f32", [False, True])
def test_room_changes_no_bit(gpu_lib, sizes, heads, kv_heads, D, f32):
    batch = Batch([o + n for o, n in sizes], 32, kv_heads, D, 94)
    want = weighed(gpu_lib, batch, batch.per, sizes, heads, D, f32, 5)
    for per in (batch.per + 90, 1000):
        got = weighed(gpu_lib, batch, per, sizes, heads, D, f32, 5)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), per


@pytest.mark.parametrize("sizes", [[(0, 512)], [(0, 300), (45, 1), (130, 70)], [(3000, 5), (0, 3), (255, 1)], [(0, 1)], [(1000, 300), (1, 700)], [(0, 0), (0, 40), (-7, 4)], [(4000, 130)]])
@pytest.mark.parametrize("heads,kv_heads,D", [(2, 2, 128), (16, 2, 64), (4, 2, 100), (6, 2, 250)])
def test_wide_tables(gpu_lib, sizes, heads, kv_heads, D):
    run_weights(gpu_lib, sizes, heads, kv_heads, D, 64, len(sizes) == 1, False, seed=6, rows=20, per=600)


@pytest.mark.parametrize("B,heads,kv_heads,D", [(1, 16, 2, 128), (3, 4, 1, 64), (2, 8, 8, 250), (40, 8, 1, 128), (1, 2048, 2048, 8)])
def test_workspaces_of_wide_tables_are_not_left(gpu_lib, B, heads, kv_heads, D):
    sizes = [(0 if b % 2 else 700, 200 + 3 * b) for b in range(B)]
    batch = Batch([o + n for o, n in sizes], 32, kv_heads, D, 95)
    table = np.full((B, 800), -1, dtype=np.int32)
    table[:, : batch.per] = batch.table
    tab, lens, starts = dev(table), dev([o + n for o, n in sizes]), dev(np.cumsum([0] + [n for _, n in sizes]))
    T = int(starts[-1])
    q = dev16(batch.queries(T, heads, D))
    need = gpu_lib.attention_weights_workspace(T, heads, D, batch.k, tab, True, gpu_lib.F32)
    room = torch.full((need + 8192,), 0xFF, dtype=torch.uint8, device="cuda")
    accs = []
    for ws in (room[4096: 4096 + need], None):
        accs.append(torch.zeros((B, kv_heads, 800 * 32), device="cuda"))
        gpu_lib.attention_prefill_weights(q, batch.k, batch.v, tab, lens, starts, accs[-1], y_dtype=gpu_lib.F32, workspace=ws)
    assert torch.equal(*accs) and torch.isfinite(accs[0]).all()
    assert (room[:4096] == 0xFF).all() and (room[4096 + need:] == 0xFF).all()
