"""Every form of the attention kernels that a head's size chooses: tiles of 64 and of 128 rows, rows that workgroups share, single tokens; and
what single tokens do on tables of more than 64 pages, without a workspace and in large batches.  The definition and the bounds are attention_ref's."""
import numpy as np
import pytest

from attention_ref import Cache, bf16
from test_gpu_attention import check_attention, dev, dev16, host, run_append, run_decode, run_prefill

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# one size at least for each built form: chunks of 32 dims that are whole (32 ... 256), and filled in part with one tile of 16 dims in the last
# chunk or two; up to 62 dims a stage is two blocks of the cache
FORMS = [2, 16, 30, 32, 40, 48, 56, 62, 64, 80, 90, 96, 98, 112, 120, 126, 128, 130, 160, 190, 192, 194, 250, 256]


@pytest.mark.parametrize("D", FORMS)
@pytest.mark.parametrize("f32", [False, True])
def test_prefill_tiles_of_128_rows(gpu_lib, D, f32):
    """A chunk of 1030 tokens behind 3200: 65 tiles a key-value head, the last of 48 rows.  Pages of three blocks, so that stages of two cross their ends."""
    run_prefill(gpu_lib, [(3200, 1030)], 64, 8, D, 96, f32, seed=21, rows=10)


@pytest.mark.parametrize("D", [32, 100, 128, 250])
@pytest.mark.parametrize("f32", [False, True])
def test_prefill_tiles_of_128_rows_of_several_sequences(gpu_lib, D, f32):
    """A prompt, an empty run, a chunk and a single token, behind rows that belong to none."""
    run_prefill(gpu_lib, [(0, 1100), (70, 0), (301, 1500), (2800, 1)], 64, 8, D, 64, f32, seed=22, rows=16, first=3, behind=2)


@pytest.mark.parametrize("D", FORMS)
@pytest.mark.parametrize("f32", [False, True])
def test_prefill_tiles_of_64_rows_and_shared_rows(gpu_lib, D, f32):
    run_prefill(gpu_lib, [(0, 70), (33, 31), (5, 0), (63, 1), (-4, 6)], 4, 2, D, 96, f32, seed=23, first=2, behind=3)
    run_prefill(gpu_lib, [(2000, 20), (0, 3), (255, 1), (256, 1)], 6, 2, D, 96, f32, seed=24, first=1, behind=2)


@pytest.mark.parametrize("D", FORMS)
@pytest.mark.parametrize("f32", [False, True])
def test_decode_of_each_form(gpu_lib, D, f32):
    run_decode(gpu_lib, [1, 33, 0, 127, 300], 6, 2, D, 96, f32, seed=25)
    run_decode(gpu_lib, [4000, 1], 18, 1, D, 96, f32, seed=26)


@pytest.mark.parametrize("D", [16, 30, 32, 62, 98, 126, 130, 190, 194])
@pytest.mark.parametrize("pairs", [False, True])
def test_append_of_each_form(gpu_lib, D, pairs):
    for f32 in (False, True):
        run_append(gpu_lib, [(0, 1), (0, 70), (5, 0), (31, 2), (33, 100), (-3, 5)], 4, 2, D, 96, f32, pairs, first=3, behind=5)
        run_append(gpu_lib, [(0, 1), (31, 1), (95, 1), (-1, 1), (200, 1)], 4, 2, D, 96, f32, pairs, one=True)


# a wave of the one workgroup has up to 64 block numbers at hand; 8192 tokens, and one more, are where it takes the next
@pytest.mark.parametrize("n", [8160, 8192, 8193, 8225, 17003, 33000])
@pytest.mark.parametrize("P,D", [(32, 64), (96, 100), (1024, 128)])
@pytest.mark.parametrize("f32", [False, True])
def test_decode_of_long_sequences_in_one_launch(gpu_lib, n, P, D, f32):
    """No workspace; tables of up to 1032 pages (64 entries of a table are taken at once where it has no more), and of 9."""
    per = -(-n // P)
    bad = [(0, p, -1) for p in (per // 2, per - 2) if 0 < p < per]
    run_decode(gpu_lib, [n, 5], 4, 2, D, P, f32, seed=27, bad=bad, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))


class Crowd:
    """Sequences of the given lengths on tables of `per` columns, of which only those that the lengths need name a page."""

    def __init__(self, lens, P, kv_heads, D, per, seed):
        self.rng, self.lens = np.random.default_rng([29, seed, D, P]), lens
        need = [-(-n // P) for n in lens]
        numbers = self.rng.permutation(sum(need) + 3).astype(np.int32)
        self.table = np.full((len(lens), per), -1, dtype=np.int32)
        self.cache = Cache(sum(need) + 3, P, kv_heads, D)
        for b, n in enumerate(lens):
            self.table[b, : need[b]], numbers = numbers[: need[b]], numbers[need[b]:]
            self.cache.put(self.table[b], 0, *(bf16(self.rng.standard_normal((n, kv_heads, D))) for _ in range(2)))
        self.k, self.v = (dev16(x) for x in self.cache.layout())


# 256 rows and more are shared only at every 8192 tokens that the tables have room for, in parts of 128 blocks at least: of three parts here, the
# sequences have three of 178 blocks, one, one and a block behind it, two and two blocks behind them, three of 128
@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (16, 4)])
@pytest.mark.parametrize("D,P", [(64, 32), (100, 96)])
@pytest.mark.parametrize("f32", [False, True])
def test_decode_of_long_sequences_among_many(gpu_lib, heads, kv_heads, D, P, f32):
    lens = [int(n) for n in np.random.default_rng(28).integers(0, 200, 70)]
    lens[3], lens[17], lens[40], lens[41], lens[69] = 17003, 4096, 4097, 8225, 12288
    crowd = Crowd(lens, P, kv_heads, D, -(-17100 // P), heads)
    crowd.table[3, crowd.table.shape[1] // 3], crowd.table[69, 5] = -1, 1 << 30
    tab = dev(crowd.table)
    assert gpu_lib.attention_workspace(len(lens), heads, D, crowd.k, tab) >= 3 * len(lens) * heads * (D + 2) * 4
    q = bf16(crowd.rng.standard_normal((len(lens), heads, D)) * 1.5)
    y = gpu_lib.attention_decode(dev16(q), crowd.k, crowd.v, tab, dev(lens), y_dtype=gpu_lib.F32 if f32 else gpu_lib.BF16)
    check_attention(host(y), q, crowd, [(b, n - 1) for b, n in enumerate(lens)], D ** -0.5, f32)
