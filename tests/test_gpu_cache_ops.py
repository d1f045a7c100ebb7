"""What a serving loop does around the paged cache -- heads that are normed and turned into it, batches that share prefixes, weights of cached tokens, eviction --
against its definition in 64 bits (cache_ref.py, attention_ref.py), with bounds derived there, on caches whose unused places hold NaN."""
import numpy as np
import pytest

from attention_ref import BF16_HALF_STEP, F32_HALF_STEP, Cache, attention, bf16
from cache_ref import evict, norm_rope, weights
from test_gpu_attention import DIMS, Batch, check_attention, dev, dev16, host, tables

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


# ---- norms, turns and the cache --------------------------------------------------------------------------------------------------
def run_norm_append(gpu_lib, sizes, heads, kv_heads, D, P, f32, pairs, rotary=None, first=0, behind=0, one=False, seed=0, shift=None, norm=True, gains=True, eps=1e-6,
                    bad=(), size=3.0, zeros=False):
    """sizes: (cached before, new) of each sequence.  Runs the call and checks q, every element of the cache and every row around."""
    rng = np.random.default_rng([13, seed, D, P, heads])
    B = len(sizes)
    per = max(1, max(-(-(o + n) // P) for o, n in sizes)) + 1
    table, pages = tables(rng, B, per)
    for b, p, value in bad:
        table[b, p] = value
    T = first + sum(n for _, n in sizes) + behind
    freq = (10000.0 ** (-np.arange(0, rotary if rotary is not None else D, 2) / D)).astype(np.float32)
    x = (rng.standard_normal((T, heads + 2 * kv_heads, D)) * size).astype(np.float32)
    if zeros:
        x[:, 0] = x[:, heads] = 0.0
    if not f32:
        x = bf16(x).astype(np.float32)
    qg, kg = [(1 + 0.3 * rng.standard_normal(D)).astype(np.float32) if gains else None for _ in range(2)]
    mark = 0.171875                                          # a bf16 that stands in every place that is not to change
    k, v = gpu_lib.kv_cache(pages, P, kv_heads, D)
    k.fill_(mark), v.fill_(mark)
    q = torch.full((T, heads, D), mark, dtype=torch.bfloat16, device="cuda")
    qkv = torch.from_numpy(x.reshape(T, -1)).cuda().to(torch.float32 if f32 else torch.bfloat16)
    start = np.cumsum([first] + [n for _, n in sizes]).astype(np.int32)
    lens = np.array([o + n for o, n in sizes], dtype=np.int32)
    as_dev = lambda a: None if a is None else dev(a, np.float32)  # noqa: E731
    got = gpu_lib.norm_rope_kv_append(qkv, as_dev(freq) if len(freq) else None, k, v, dev(table), dev(lens), heads, as_dev(qg), as_dev(kg), eps,
                                      q_start=None if one else dev(start), pairs=pairs, norm=norm, shift=None if shift is None else dev(shift), q=q)
    torch.cuda.synchronize()
    assert got is q
    cache = Cache(pages, P, kv_heads, D, fill=mark)
    want_q, off_q = np.full((T, heads, D), mark), np.zeros((T, heads, D))
    off_k = np.zeros_like(cache.k, dtype=np.float64)
    for b, (old, new) in enumerate(sizes):
        r = slice(int(start[b]), int(start[b]) + new)
        pos = np.arange(old, old + new)
        at = pos + (0 if shift is None else shift[b])
        y, off = norm_rope(x[r, :heads].astype(np.float64), at, freq, pairs, qg, eps, norm)
        want_q[r], off_q[r] = y, off * (1 + BF16_HALF_STEP) + BF16_HALF_STEP * np.abs(y)
        y, off = norm_rope(x[r, heads:heads + kv_heads].astype(np.float64), at, freq, pairs, kg, eps, norm)
        off = off * (1 + BF16_HALF_STEP) + BF16_HALF_STEP * np.abs(y)
        for i in np.nonzero(pos >= 0)[0]:
            page, to = table[b][pos[i] // P], pos[i] % P
            if 0 <= page < pages:
                cache.k[page, to], off_k[page, to] = y[i], off[i]
                cache.v[page, to] = bf16(x[r, heads + kv_heads:][i])
    assert np.all(np.abs(host(q) - want_q) <= off_q)
    gk, gv = cache.from_layout(host(k), host(v))
    # the reference's keys are held in fp32: a step of that on top
    assert np.all(np.abs(gk - cache.k) <= off_k + 2 ** -23 * np.abs(cache.k) * (off_k > 0))
    assert np.array_equal(gv, cache.v.astype(np.float64))
    if D % 8:                                                # dims behind the head's end: zeros in the keys of stored tokens
        pad = host(k)[:, :, :, -1, :, D % 8:]
        written = gk[..., -1] != mark
        assert set(np.unique(pad)) <= {0.0, mark} and (not written.any() or (pad == 0.0).sum() >= written.sum() * (8 - D % 8))


@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("pairs", [False, True])
def test_norm_append_single_tokens(gpu_lib, D, pairs):
    sizes = [(0, 1), (1, 1), (31, 1), (32, 1), (95, 1), (96, 1), (-1, 1), (200, 1)]
    run_norm_append(gpu_lib, sizes, 6, 3, D, 96, D % 3 == 0, pairs, one=True)


@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("pairs", [False, True])
def test_norm_append_runs(gpu_lib, D, pairs):
    sizes = [(0, 1), (0, 70), (5, 0), (31, 2), (17, 14), (40, 24), (0, 0), (33, 100), (-3, 5)]
    run_norm_append(gpu_lib, sizes, 4, 2, D, 64, D % 3 != 0, pairs, first=3, behind=5)


@pytest.mark.parametrize("one", [False, True])
@pytest.mark.parametrize("rotary,D", [(0, 64), (2, 64), (32, 128), (24, 100), (98, 100), (2, 256), (2, 250), (14, 90), (240, 250), (16, 256)])
def test_norm_append_turns_the_first_dims_alone(gpu_lib, one, rotary, D):
    sizes = [(3, 1), (70, 1)] if one else [(3, 40), (70, 1)]
    for pairs in (False, True):
        run_norm_append(gpu_lib, sizes, 2, 1, D, 32, True, pairs, rotary=rotary, one=one)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (7, 1), (64, 8), (40, 40)])
@pytest.mark.parametrize("f32", [False, True])
def test_norm_append_head_layouts_and_many_blocks(gpu_lib, heads, kv_heads, f32):
    run_norm_append(gpu_lib, [(9, 700), (0, 513)], heads, kv_heads, 128, 256, f32, False)
    run_norm_append(gpu_lib, [(i * 13, 1) for i in range(40)], heads, kv_heads, 128, 256, f32, False, one=True)


@pytest.mark.parametrize("one", [False, True])
@pytest.mark.parametrize("options", [dict(shift=[0, 1000, -30, 2 ** 31 - 1]), dict(norm=False, shift=[7, 0, 123456, 5]), dict(norm=False), dict(gains=False),
                                     dict(eps=0.0, zeros=True), dict(eps=1e3), dict(size=1e30), dict(size=1e-25, eps=0.0), dict(bad=[(0, 1, -1), (1, 0, 1 << 30), (3, 2, -2 ** 31)])])
def test_norm_append_options(gpu_lib, one, options):
    sizes = [(40, 1), (10, 1), (0, 1), (70, 1)] if one else [(0, 90), (10, 60), (0, 1), (3, 70)]
    for D, pairs in [(64, False), (100, False), (100, True)]:
        run_norm_append(gpu_lib, sizes, 4, 2, D, 32, True, pairs, one=one, seed=1, **options)


@pytest.mark.parametrize("one", [False, True])
@pytest.mark.parametrize("D", [64, 100, 128])
@pytest.mark.parametrize("f32", [False, True])
def test_without_a_norm_it_is_the_plain_append(gpu_lib, one, D, f32):
    rng = np.random.default_rng(D)
    x = torch.from_numpy(rng.standard_normal((90, 8 * D)).astype(np.float32)).cuda().to(torch.float32 if f32 else torch.bfloat16)
    x = x[:2].contiguous() if one else x
    freq, table, lens, start = dev((10000.0 ** (-np.arange(0, D, 2) / D)).astype(np.float32), np.float32), dev([[3, 1], [0, 2]]), dev([80, 50]), None if one else dev([0, 60, 90])
    (k0, v0), (k1, v1) = gpu_lib.kv_cache(4, 64, 2, D), gpu_lib.kv_cache(4, 64, 2, D)
    q0 = gpu_lib.rope_kv_append(x, freq, k0, v0, table, lens, 4, q_start=start)
    q1 = gpu_lib.norm_rope_kv_append(x, freq, k1, v1, table, lens, 4, q_start=start, norm=False)
    for a, b in ((q0, q1), (k0, k1), (v0, v1)):
        assert torch.equal(a, b)


# ---- shared prefixes ----------------------------------------------------------------------------------------------------------------
class Shared(Batch):
    """Sequences of the given lengths in groups: group i, of counts[i] sequences, shares its first prefixes[i] tokens; what the others' own tables name
    for these are pages of NaN."""

    def __init__(self, lens, counts, prefixes, P, kv_heads, D, seed=0, before=0, per=None):
        super().__init__([max(n, 0) for n in lens], P, kv_heads, D, seed, per)
        self.lens = list(lens)
        self.start = np.cumsum([before] + list(counts)).astype(np.int32)
        self.prefix = np.array(prefixes, dtype=np.int32)
        first_of = {}
        for i, n in enumerate(counts):
            s = int(self.start[i])
            for b in range(s, s + n):
                first_of[b] = (s, max(0, min(int(prefixes[i]), self.per * P)))
        for b, (s, n) in first_of.items():                  # the prefix in full on the first one's pages, nothing on the others'
            if b == s and n:
                k, v = (bf16(self.rng.standard_normal((n, kv_heads, D))) for _ in range(2))
                self.cache.put(self.table[b], 0, k, v)
            elif n:
                self.cache.put(self.table[b], 0, *[np.full((n, kv_heads, D), np.nan)] * 2)
        self.first_of = first_of
        k, v = self.cache.layout()
        self.k, self.v = dev16(k), dev16(v)

    def keys_of(self, b):
        n = max(0, min(self.lens[b], self.per * self.cache.P))
        k, v, there = self.cache.get(self.table[b], n)
        s, shared = self.first_of.get(b, (b, 0))
        shared = min(shared, n)
        if shared:
            fk, fv, ft = self.cache.get(self.table[s], shared)
            k, v, there = (np.concatenate([f, x[shared:]]) for f, x in ((fk, k), (fv, v), (ft, there)))
        return k, v, there


def run_shared(gpu_lib, lens, counts, prefixes, heads, kv_heads, D, P, f32, seed=0, before=0, bad=(), scale=None, std=1.5, rows=None, per=None, **more):
    batch = Shared(lens, counts, prefixes, P, kv_heads, D, seed, before, per)
    for b, p, value in bad:
        batch.table[b, p] = value
    B = len(lens)
    q = batch.queries(B, heads, D, std)
    y = gpu_lib.attention_decode_shared(dev16(q), batch.k, batch.v, dev(batch.table), dev(lens), dev(batch.start), dev(batch.prefix), scale,
                                        gpu_lib.F32 if f32 else gpu_lib.BF16, **more)
    assert y.shape == (B, heads * D)
    got = host(y).reshape(B, heads, D)
    picked = range(B) if rows is None else sorted({0, B - 1} | set(int(i) for i in batch.rng.integers(0, B, rows)))
    for b in picked:
        k, v, there = batch.keys_of(b)
        o, bounds = attention(q[b], np.where(there[:, None, None], k, 0), np.where(there[:, None, None], v, 0), there, scale or D ** -0.5)
        off = np.abs(got[b] - o)
        assert np.all(off <= bounds[1 if f32 else 0]), (b, float(np.nanmax(off)), float(np.nanmax(off / bounds[1 if f32 else 0])), bool(np.isnan(off).any()))


@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("f32", [False, True])
def test_shared_dims(gpu_lib, D, f32):
    run_shared(gpu_lib, [70, 71, 95, 96, 97, 130, 40, 69, 300], [6, 2], [70, 33], 6, 2, D, 96, f32)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (5, 5), (8, 1), (16, 1), (17, 1), (33, 1), (64, 8), (96, 2)])
@pytest.mark.parametrize("f32", [False, True])
def test_shared_head_layouts(gpu_lib, heads, kv_heads, f32):
    run_shared(gpu_lib, [200, 131, 140, 400, 132, 133, 160], [4, 1, 2], [131, 77, 100], heads, kv_heads, 128, 32, f32, seed=1)


# prefixes of no tokens, that end inside a block and page, at their ends, and behind the end of a sequence; sequences without any tokens or in no group
@pytest.mark.parametrize("lens,counts,prefixes,before", [
    ([1], [1], [1], 0), ([0], [1], [0], 0), ([0, 0], [2], [64], 0), ([5, 9], [2], [0], 0), ([64, 64, 64], [3], [64], 0), ([65, 64, 63, 1, 0, 96], [6], [64], 0),
    ([100, 50, 33, 32, 31, 500], [2, 2], [40, 33], 1), ([100, 100, 100], [1, 1, 1], [99, 100, 101], 0), ([50, 50], [0, 2, 0], [7, 30, 9], 0),
    ([3000, 2999, 3100, 0, 2000], [5], [2999], 0), ([5000, 40, 70], [2], [32], 1), ([2048] * 3, [3], [1024], 0), ([900] * 70, [70], [700], 0),
    ([90, 91, 92], [3], [-5], 0), ([90, 91, 92], [3], [2 ** 31 - 1], 0)])
@pytest.mark.parametrize("heads,kv_heads,D", [(4, 1, 128), (3, 3, 64), (16, 2, 100)])
def test_shared_lengths(gpu_lib, lens, counts, prefixes, before, heads, kv_heads, D):
    run_shared(gpu_lib, lens, counts, prefixes, heads, kv_heads, D, 64, len(lens) % 2 == 0, seed=2, before=before, rows=9)


def test_shared_leaves_out_pages_that_are_not_there(gpu_lib):
    run_shared(gpu_lib, [400, 410, 420], [3], [300], 4, 2, 64, 64, True, seed=3, bad=[(0, 1, -1), (0, 4, 1 << 30), (1, 5, -2 ** 31), (2, 6, 2 ** 31 - 1), (1, 0, 1 << 30)])


@pytest.mark.parametrize("scale,std", [(1.0, 3.0), (1e-3, 1.0), (0.7, 0.0), (20.0, 4.0)])
def test_shared_peaked_and_flat_weights(gpu_lib, scale, std):
    run_shared(gpu_lib, [700, 745, 1500], [3], [650], 4, 2, 128, 64, True, seed=4, scale=scale, std=std)


def test_shared_many_sequences_and_wide_tables(gpu_lib):
    rng = np.random.default_rng(8)
    lens = [int(n) for n in rng.integers(100, 400, 300)]
    run_shared(gpu_lib, lens, [100, 30, 170], [100, 99, 37], 8, 2, 64, 32, True, seed=5, rows=12)
    run_shared(gpu_lib, [120, 130], [2], [100], 8, 2, 64, 32, False, seed=5, per=600)


# ---- weights of cached tokens ---------------------------------------------------------------------------------------------------------
def run_weights(gpu_lib, sizes, heads, kv_heads, D, P, f32, one, seed=0, first=0, behind=0, per=None, scale=None, std=1.5, bad=(), rows=None, room=0, **more):
    """sizes: (cached before, new); checks the attention, every accumulator, and that those behind a sequence's tokens stay."""
    lens = [o + n for o, n in sizes]
    batch = Batch([max(n, 0) for n in lens], P, kv_heads, D, seed, per)
    for b, p, value in bad:
        batch.table[b, p] = value
    B, C = len(sizes), batch.per * P + room
    T = first + sum(n for _, n in sizes) + behind
    q = batch.queries(T, heads, D, std)
    start = np.cumsum([first] + [n for _, n in sizes])
    old = np.abs(batch.rng.standard_normal((B, kv_heads, C))).astype(np.float32)
    old_dev = torch.from_numpy(old).cuda()
    for b, (o, n) in enumerate(sizes):                       # new tokens begin with nothing, whatever stands there
        old_dev[b, :, max(o, 0): max(o + n, 0)] = float("nan")
    scale_, t = scale or D ** -0.5, gpu_lib.F32 if f32 else gpu_lib.BF16
    if one:
        y = gpu_lib.attention_decode_weights(dev16(q), batch.k, batch.v, dev(batch.table), dev(lens), old_dev, scale, t, **more)
    else:
        y = torch.full((T, heads * D), 7.25, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
        y = gpu_lib.attention_prefill_weights(dev16(q), batch.k, batch.v, dev(batch.table), dev(lens), dev(start), old_dev, scale, t, y=y, **more)
        assert np.all(host(y)[:first] == 7.25) and np.all(host(y)[T - behind:] == 7.25)
    at = [(b, o + i) for b, (o, n) in enumerate(sizes) for i in range(n)]
    picked = range(len(at)) if rows is None else sorted({0, len(at) - 1} | set(int(i) for i in batch.rng.integers(0, len(at), rows)))
    check_attention(host(y)[[first + i for i in picked]], q[[first + i for i in picked]], batch, [at[i] for i in picked], scale_, f32, "D %d" % D)
    got = host(old_dev)
    for b, (o, n) in enumerate(sizes):
        end = max(lens[b], 0)
        k, _, there = batch.cache.get(batch.table[b], end)
        k = np.where(there[:, None, None], k, 0)
        want, off = np.zeros((kv_heads, end)), np.zeros((kv_heads, end))
        want[:, : max(o, 0)] = old[b, :, : max(o, 0)]
        for i in range(n):
            w, e = weights(q[start[b] + i], k, there & (np.arange(end) <= o + i), scale_)
            want, off = want + w, off + e
        off = off + (n * heads // kv_heads + 2) * F32_HALF_STEP * want
        assert np.all(np.abs(got[b, :, :end] - want) <= off), (b, float(np.nanmax(np.abs(got[b, :, :end] - want) / (off + 1e-38))), bool(np.isnan(got[b, :, :end]).any()))
        assert np.array_equal(got[b, :, end:], old[b, :, end:].astype(np.float64))


LENS = [1, 2, 31, 32, 33, 64, 0, 127, 129, 300]


@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("f32", [False, True])
def test_decode_weights_dims(gpu_lib, D, f32):
    run_weights(gpu_lib, [(n - 1, 1) for n in LENS], 6, 2, D, 96, f32, True)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (5, 5), (8, 1), (17, 1), (33, 1), (150, 2), (64, 8)])
@pytest.mark.parametrize("f32", [False, True])
def test_decode_weights_head_layouts(gpu_lib, heads, kv_heads, f32):
    run_weights(gpu_lib, [(n - 1, 1) for n in LENS], heads, kv_heads, 128, 32, f32, True, seed=1, room=5)


@pytest.mark.parametrize("lens,per", [([1], 1), ([0], 1), ([0, 0, 0], 40), ([5000], None), ([1, 9000], None), ([4097, 1, 2050, 0, 777], 200), ([2048] * 3, None), ([33], 500)])
@pytest.mark.parametrize("heads,kv_heads,D", [(4, 1, 128), (3, 3, 64), (16, 2, 100)])
def test_decode_weights_lengths(gpu_lib, lens, per, heads, kv_heads, D):
    run_weights(gpu_lib, [(n - 1, 1) for n in lens], heads, kv_heads, D, 64, len(lens) % 2 == 0, True, seed=2, per=per)


@pytest.mark.parametrize("scale,std", [(1.0, 3.0), (1e-3, 1.0), (0.7, 0.0), (20.0, 4.0)])
@pytest.mark.parametrize("f32", [False, True])
def test_weights_peaked_and_flat(gpu_lib, scale, std, f32):
    run_weights(gpu_lib, [(3000, 1), (44, 1)], 4, 2, 128, 64, f32, True, seed=4, scale=scale, std=std)
    run_weights(gpu_lib, [(0, 100), (44, 3)], 4, 2, 128, 64, f32, False, seed=4, scale=scale, std=std)
    run_weights(gpu_lib, [(3000, 5)], 4, 2, 64, 64, f32, False, seed=4, scale=scale, std=std)


def test_weights_leave_out_pages_that_are_not_there(gpu_lib):
    bad = [(0, 1, -1), (1, 1, 1 << 30), (2, 0, -2 ** 31), (3, 7, 2 ** 31 - 1), (3, 46, -3)]
    run_weights(gpu_lib, [(199, 1), (99, 1), (63, 1), (2999, 1)], 4, 2, 64, 64, True, True, seed=5, bad=bad)
    run_weights(gpu_lib, [(100, 100), (0, 100), (60, 4), (2900, 100)], 4, 2, 64, 64, True, False, seed=5, bad=bad, rows=40)


@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("f32", [False, True])
def test_prefill_weights_dims(gpu_lib, D, f32):
    run_weights(gpu_lib, [(0, 70), (33, 31), (5, 0), (63, 1), (0, 1), (-4, 6), (0, 300)], 4, 2, D, 32, f32, False, first=2, behind=3, rows=60)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 3), (7, 1), (12, 1), (64, 8), (65, 1)])
@pytest.mark.parametrize("f32", [False, True])
def test_prefill_weights_head_layouts(gpu_lib, heads, kv_heads, f32):
    run_weights(gpu_lib, [(10, 40), (0, 129), (100, 3)], heads, kv_heads, 128, 96, f32, False, seed=1, rows=40, room=7)


@pytest.mark.parametrize("sizes", [[(0, 1)], [(0, 0), (3, 1)], [(0, 64)], [(0, 65)], [(0, 127), (0, 128)], [(4000, 1)], [(4000, 17)], [(0, 1030)], [(63, 1), (64, 1), (65, 2)],
                                   [(1000, 300), (1, 700)], [(3000, 5), (0, 3), (255, 1)], [(-2, 4), (1100, 2)], [(-7, 4), (0, 40)]])
@pytest.mark.parametrize("heads,kv_heads,D", [(2, 2, 128), (8, 1, 64), (4, 2, 100)])
def test_prefill_weights_lengths(gpu_lib, sizes, heads, kv_heads, D):
    run_weights(gpu_lib, sizes, heads, kv_heads, D, 64, len(sizes) == 1, False, seed=2, rows=40)


# ---- eviction ------------------------------------------------------------------------------------------------------------------------------
def make_weights(rng, shape, kind):
    w = np.exp(2 * rng.standard_normal(shape)).astype(np.float32)
    if kind == "ties":
        w = np.round(w * 2) / 2
    elif kind == "equal":
        w[:] = 0.25
    elif kind == "signs":                                    # whatever a caller's arithmetic left there
        w = (rng.standard_normal(shape) * np.exp(20 * rng.standard_normal(shape))).astype(np.float32)
        w[rng.random(shape) < 0.2] = -0.0
        w[rng.random(shape) < 0.2] = 0.0
        w[rng.random(shape) < 0.05] = np.nan
        w[rng.random(shape) < 0.05] = -np.nan
        w[rng.random(shape) < 0.05] = np.inf
        w[rng.random(shape) < 0.05] = -np.inf
    elif kind == "zeros":
        w[rng.random(shape) < 0.9] = 0.0
    return w.astype(np.float32)


def run_evict(gpu_lib, lens, kv_heads, D, P, keep, recent, kind="ties", seed=0, per=None, bad=(), bad_out=(), in_place=False, room=0):
    batch = Batch(lens, P, kv_heads, D, seed, per)
    rng, B = batch.rng, len(lens)
    for b, p, value in bad:
        batch.table[b, p] = value
    cap = batch.per * P
    per_out = -(-min(keep, cap) // P)
    old_pages = batch.cache.pages
    cache = Cache(old_pages + B * per_out + 1, P, kv_heads, D, fill=0.34375)     # new pages hold something that is to stay
    cache.k[:old_pages], cache.v[:old_pages] = batch.cache.k, batch.cache.v
    out = (old_pages + rng.permutation(B * per_out + 1)[: B * per_out]).reshape(B, per_out).astype(np.int32)
    for b, p, value in bad_out:
        out[b, p] = value
    k, v = cache.layout()
    k, v = dev16(k), dev16(v)
    w = make_weights(rng, (B, kv_heads, cap + room), kind)
    wd, kv_len = torch.from_numpy(w).cuda(), dev(lens)
    kept = torch.full((B, kv_heads, keep), -7, dtype=torch.int32, device="cuda")
    w_out = wd if in_place else torch.full((B, kv_heads, max(per_out * P, keep if keep < cap else cap) + room), 9.5, dtype=torch.float32, device="cuda")
    before = host(w_out)
    got = gpu_lib.kv_evict(k, v, dev(batch.table), kv_len, wd, keep, recent, dev(out), kv_len_out=kv_len if in_place else None, weights_out=w_out, kept=kept)
    assert got[1] is w_out and got[2] is kept and (got[0] is kv_len or not in_place)
    want_len = np.array([min(max(n, 0), keep) for n in lens])
    assert np.array_equal(got[0].cpu().numpy(), want_len)
    want_w, got_kept, want_kept = before.copy(), kept.cpu().numpy(), np.full((B, kv_heads, keep), -7)
    for b, n in enumerate(lens):
        for h in range(kv_heads):
            at = evict(w[b, h], n, keep, recent)
            want_kept[b, h, : len(at)] = at
            want_w[b, h, : len(at)] = w[b, h, at]
            for i, p in enumerate(at):
                page, to = batch.table[b, p // P], out[b, i // P]
                if 0 <= to < cache.pages:
                    there = 0 <= page < cache.pages
                    cache.k[to, i % P, h] = cache.k[page, p % P, h] if there else 0
                    cache.v[to, i % P, h] = cache.v[page, p % P, h] if there else 0
    assert np.array_equal(got_kept, want_kept)
    assert np.array_equal(host(w_out).astype(np.float32).view(np.int32) & 0x7FFFFFFF, want_w.astype(np.float32).view(np.int32) & 0x7FFFFFFF)
    gk, gv = cache.from_layout(host(k), host(v))
    assert np.array_equal(gk, cache.k, equal_nan=True) and np.array_equal(gv, cache.v, equal_nan=True)


@pytest.mark.parametrize("D", DIMS)
def test_evict_dims(gpu_lib, D):
    run_evict(gpu_lib, [200, 61, 60, 59, 0, 1, 90], 3, D, 32, 60, 11)


@pytest.mark.parametrize("kind", ["ties", "equal", "signs", "zeros", "any"])
@pytest.mark.parametrize("keep,recent", [(1, 0), (1, 1), (31, 0), (32, 32), (33, 5), (100, 1), (257, 256), (499, 0), (500, 100), (5000, 17)])
def test_evict_budgets_and_weights(gpu_lib, kind, keep, recent):
    run_evict(gpu_lib, [500, 33, 257, 2, 501], 2, 64, 64, keep, recent, kind=kind, seed=1, room=3)


@pytest.mark.parametrize("kind", ["ties", "equal", "zeros"])
@pytest.mark.parametrize("keep,recent", [(4000, 300), (9000, 0), (100, 50)])
def test_evict_long(gpu_lib, kind, keep, recent):
    run_evict(gpu_lib, [20000, 9001, 4096, 4097], 1, 8, 256, keep, recent, kind=kind, seed=2)


@pytest.mark.parametrize("kind", ["ties", "equal", "any"])
def test_evict_in_place_of_lengths_and_weights(gpu_lib, kind):
    run_evict(gpu_lib, [9000, 300, 5000, 77], 2, 16, 64, 120, 30, kind=kind, seed=3, in_place=True)
    run_evict(gpu_lib, [9000, 300, 5000, 77], 2, 16, 64, 6000, 30, kind=kind, seed=3, in_place=True)


def test_evict_pages_that_are_not_there(gpu_lib):
    run_evict(gpu_lib, [300, 200, 40], 2, 24, 32, 100, 20, seed=4, bad=[(0, 1, -1), (1, 0, 1 << 30), (2, 0, -2 ** 31)], bad_out=[(0, 1, -1), (1, 2, 1 << 30), (2, 0, 2 ** 31 - 1)])


def test_evict_many_sequences(gpu_lib):
    rng = np.random.default_rng(5)
    run_evict(gpu_lib, [int(n) for n in rng.integers(0, 200, 150)], 3, 8, 32, 64, 8, seed=5, per=20)
