"""The attention half of a decoder layer -- rotary positions into a paged cache, attention of single tokens and of runs of them over it --
against its definition in 64 bits (attention_ref.py), with bounds derived there, on caches whose unused places hold NaN."""
import numpy as np
import pytest

import oracle
from attention_ref import BF16_HALF_STEP, Cache, attention, bf16, rope
from paper_2402_17764_amd import synth

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def dev16(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(torch.bfloat16)


def dev(a, dt=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dt)).cuda()


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def tables(rng, B, per, spare=3):
    """Page tables of B sequences of `per` pages each, all pages different, in random order: (table [B, per], number of pages)."""
    pages = B * per + spare
    return rng.permutation(pages)[: B * per].reshape(B, per).astype(np.int32), pages


class Batch:
    """Sequences of the given lengths with random keys and values in a cache of NaN."""

    def __init__(self, lens, P, kv_heads, D, seed=0, per=None, scale=1.0):
        self.rng = np.random.default_rng([7, seed, D, P, kv_heads, len(lens)])
        self.lens = list(lens)
        self.per = per or max(1, -(-max(self.lens) // P))
        self.table, pages = tables(self.rng, len(lens), self.per)
        self.cache = Cache(pages, P, kv_heads, D)
        for b, n in enumerate(self.lens):
            k, v = (bf16(self.rng.standard_normal((n, kv_heads, D)) * s) for s in (scale, 1.0))
            self.cache.put(self.table[b], 0, k, v)
        k, v = self.cache.layout()
        self.k, self.v = dev16(k), dev16(v)

    def queries(self, T, heads, D, std=1.5):
        return bf16(self.rng.standard_normal((T, heads, D)) * std)


def check_attention(got, q, batch, rows, scale, f32, label=""):
    """rows: (sequence, position) of each row of q; got [T, heads D] on the host."""
    heads, D = q.shape[1:]
    for t, (b, pos) in enumerate(rows):
        k, v, there = batch.cache.get(batch.table[b], max(batch.lens[b], 0))
        there = there & (np.arange(len(there)) <= pos)
        o, bounds = attention(q[t], np.where(there[:, None, None], k, 0), np.where(there[:, None, None], v, 0), there, scale)
        off = np.abs(got[t].reshape(heads, D) - o)
        assert np.all(off <= bounds[1 if f32 else 0]), (label, t, b, pos, float(np.nanmax(off)), float((off / bounds[1 if f32 else 0]).max()), bool(np.isnan(off).any()))


DIMS = [2, 8, 24, 40, 56, 64, 80, 90, 96, 100, 120, 128, 160, 192, 250, 256]


# ---- rotary positions and the cache -----------------------------------------------------------------------------------------
def run_append(gpu_lib, sizes, heads, kv_heads, D, P, f32, pairs, rotary=None, first=0, behind=0, one=False, seed=0, bad=()):
    """sizes: (cached before, new) of each sequence.  Runs the call and checks q, every element of the cache and every row around."""
    rng = np.random.default_rng([11, seed, D, P, heads])
    B = len(sizes)
    per = max(1, max(-(-(o + n) // P) for o, n in sizes)) + 1
    table, pages = tables(rng, B, per)
    for b, p, value in bad:
        table[b, p] = value
    T = first + sum(n for _, n in sizes) + behind
    freq = (10000.0 ** (-np.arange(0, rotary if rotary is not None else D, 2) / D)).astype(np.float32)
    x = rng.standard_normal((T, heads + 2 * kv_heads, D)).astype(np.float32)
    if not f32:
        x = bf16(x).astype(np.float32)
    mark = 0.171875                                          # a bf16 that stands in every place that is not to change
    k, v = gpu_lib.kv_cache(pages, P, kv_heads, D)
    k.fill_(mark), v.fill_(mark)
    q = torch.full((T, heads, D), mark, dtype=torch.bfloat16, device="cuda")
    qkv = torch.from_numpy(x.reshape(T, -1)).cuda().to(torch.float32 if f32 else torch.bfloat16)
    start = np.cumsum([first] + [n for _, n in sizes]).astype(np.int32)
    lens = np.array([o + n for o, n in sizes], dtype=np.int32)
    got = gpu_lib.rope_kv_append(qkv, dev(freq, np.float32) if len(freq) else None, k, v, dev(table), dev(lens), heads,
                                 q_start=None if one else dev(start), pairs=pairs, q=q)
    torch.cuda.synchronize()
    assert got is q
    cache = Cache(pages, P, kv_heads, D, fill=mark)
    want_q, off_q = np.full((T, heads, D), mark), np.zeros((T, heads, D))
    off_k = np.zeros_like(cache.k, dtype=np.float64)
    for b, (old, new) in enumerate(sizes):
        r = slice(int(start[b]), int(start[b]) + new)
        pos = np.arange(old, old + new)
        y, off = rope(x[r, : heads + kv_heads].astype(np.float64), pos, freq, pairs)
        off = off * (1 + BF16_HALF_STEP) + BF16_HALF_STEP * np.abs(y)
        want_q[r], off_q[r] = y[:, :heads], off[:, :heads]
        stored = pos >= 0
        for i in np.nonzero(stored)[0]:
            page, at = table[b][pos[i] // P], pos[i] % P
            if 0 <= page < pages:
                cache.k[page, at], off_k[page, at] = y[i, heads:], off[i, heads:]
                cache.v[page, at] = bf16(x[r, heads + kv_heads:][i])
    assert np.all(np.abs(host(q) - want_q) <= off_q)
    gk, gv = cache.from_layout(host(k), host(v))
    # the reference's keys are held in fp32: a step of that on top
    assert np.all(np.abs(gk - cache.k) <= off_k + 2 ** -23 * np.abs(cache.k) * (off_k > 0))
    assert np.array_equal(gv, cache.v.astype(np.float64))
    if D % 8:                                                # dims behind the head's end: zeros in the keys of stored tokens
        pad = host(k)[:, :, :, -1, :, D % 8:]
        written = cache.from_layout(host(k), host(v))[0][..., -1] != mark
        assert set(np.unique(pad)) <= {0.0, mark} and (not written.any() or (pad == 0.0).sum() >= written.sum() * (8 - D % 8))


@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("pairs", [False, True])
def test_append_single_tokens(gpu_lib, D, pairs):
    sizes = [(0, 1), (1, 1), (31, 1), (32, 1), (95, 1), (96, 1), (-1, 1), (200, 1)]
    run_append(gpu_lib, sizes, 6, 3, D, 96, D % 3 == 0, pairs, one=True)


@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("pairs", [False, True])
def test_append_runs(gpu_lib, D, pairs):
    sizes = [(0, 1), (0, 70), (5, 0), (31, 2), (17, 14), (40, 24), (0, 0), (33, 100), (-3, 5)]
    run_append(gpu_lib, sizes, 4, 2, D, 64, D % 3 != 0, pairs, first=3, behind=5)


@pytest.mark.parametrize("one", [False, True])
@pytest.mark.parametrize("rotary,D", [(0, 64), (2, 64), (32, 128), (24, 100), (98, 100), (2, 256), (2, 250), (14, 90), (240, 250)])
def test_append_turns_the_first_dims_alone(gpu_lib, one, rotary, D):
    sizes = [(3, 1), (70, 1)] if one else [(3, 40), (70, 1)]
    for pairs in (False, True):
        run_append(gpu_lib, sizes, 2, 1, D, 32, True, pairs, rotary=rotary, one=one)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (7, 1), (64, 8), (40, 40)])
@pytest.mark.parametrize("f32", [False, True])
def test_append_head_layouts_and_many_blocks(gpu_lib, heads, kv_heads, f32):
    run_append(gpu_lib, [(9, 700), (0, 513)], heads, kv_heads, 128, 256, f32, False)
    run_append(gpu_lib, [(i * 13, 1) for i in range(40)], heads, kv_heads, 128, 256, f32, False, one=True)


def test_append_far_positions(gpu_lib):
    """Angles of hundreds of thousands of turns.  The table's pages are mostly not there: one page is enough."""
    D, P, heads = 128, 32, 2
    freq = (10000.0 ** (-np.arange(0, D, 2) / D)).astype(np.float32)
    rng = np.random.default_rng(3)
    for one, pos in [(True, 3_000_001), (False, 7_654_321)]:
        n = 1 if one else 40
        per = (pos + n) // P + 1
        table = np.full((1, per), -1, dtype=np.int32)
        table[0, pos // P] = 0
        x = bf16(rng.standard_normal((n, heads + 2, D)))
        k, v = gpu_lib.kv_cache(1, P, 1, D)
        q = gpu_lib.rope_kv_append(dev16(x.reshape(n, -1)), dev(freq, np.float32), k, v, dev(table), dev([pos + n]), heads, q_start=None if one else dev([0, n]))
        y, off = rope(x[:, :heads], np.arange(pos, pos + n), freq, False)
        assert np.all(np.abs(host(q) - y) <= off * 1.01 + BF16_HALF_STEP * np.abs(y))


def test_append_leaves_out_pages_that_are_not_there(gpu_lib):
    for one in (False, True):
        sizes = [(40, 1), (10, 1), (70, 1)] if one else [(0, 90), (10, 60), (3, 5)]
        run_append(gpu_lib, sizes, 2, 2, 64, 32, False, False, one=one, bad=[(0, 1, -1), (1, 0, 1 << 30), (2, 2, -2 ** 31)])


# ---- single tokens ----------------------------------------------------------------------------------------------------------
def run_decode(gpu_lib, lens, heads, kv_heads, D, P, f32, seed=0, per=None, scale=None, bad=(), std=1.5, workspace=None):
    batch = Batch(lens, P, kv_heads, D, seed, per)
    for b, p, value in bad:
        batch.table[b, p] = value
    q = batch.queries(len(lens), heads, D, std)
    y = gpu_lib.attention_decode(dev16(q), batch.k, batch.v, dev(batch.table), dev(lens), scale, gpu_lib.F32 if f32 else gpu_lib.BF16, workspace=workspace)
    assert y.shape == (len(lens), heads * D)
    check_attention(host(y), q, batch, [(b, n - 1) for b, n in enumerate(lens)], scale or D ** -0.5, f32, "D %d" % D)


LENS = [1, 2, 31, 32, 33, 64, 0, 127, 129, 300]


@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("f32", [False, True])
def test_decode_dims(gpu_lib, D, f32):
    run_decode(gpu_lib, LENS, 6, 2, D, 96, f32)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (5, 5), (8, 1), (16, 1), (17, 1), (33, 1), (64, 8), (96, 2)])
@pytest.mark.parametrize("f32", [False, True])
def test_decode_head_layouts(gpu_lib, heads, kv_heads, f32):
    run_decode(gpu_lib, LENS, heads, kv_heads, 128, 32, f32, seed=1)


@pytest.mark.parametrize("lens,per", [([1], 1), ([0], 1), ([0, 0, 0], 40), ([5000], None), ([1, 9000], None), ([4097, 1, 2050, 0, 777], 200), ([2048] * 3, None), ([33], 500)])
@pytest.mark.parametrize("heads,kv_heads,D", [(4, 1, 128), (3, 3, 64), (16, 2, 100)])
def test_decode_lengths(gpu_lib, lens, per, heads, kv_heads, D):
    run_decode(gpu_lib, lens, heads, kv_heads, D, 64, len(lens) % 2 == 0, seed=2, per=per)


@pytest.mark.parametrize("B", [65, 130, 700])
def test_decode_many_sequences(gpu_lib, B):
    rng = np.random.default_rng(B)
    run_decode(gpu_lib, [int(n) for n in rng.integers(0, 200, B)], 4, 2, 64, 32, True, seed=3, per=30)


@pytest.mark.parametrize("scale,std", [(1.0, 3.0), (1e-3, 1.0), (0.7, 0.0), (20.0, 4.0)])
def test_decode_peaked_and_flat_weights(gpu_lib, scale, std):
    run_decode(gpu_lib, [700, 45], 4, 2, 128, 64, True, seed=4, scale=scale, std=std)


def test_decode_leaves_out_pages_that_are_not_there(gpu_lib):
    run_decode(gpu_lib, [200, 100, 64, 3000], 4, 2, 64, 64, True, seed=5, bad=[(0, 1, -1), (1, 1, 1 << 30), (2, 0, -2 ** 31), (3, 7, 2 ** 31 - 1), (3, 46, -3)])


# ---- runs of tokens ----------------------------------------------------------------------------------------------------------
def run_prefill(gpu_lib, sizes, heads, kv_heads, D, P, f32, seed=0, first=0, behind=0, per=None, rows=None, workspace=None, scale=None, std=1.5):
    lens = [o + n for o, n in sizes]
    batch = Batch([max(n, 0) for n in lens], P, kv_heads, D, seed, per)
    T = first + sum(n for _, n in sizes) + behind
    q = batch.queries(T, heads, D, std)
    start = np.cumsum([first] + [n for _, n in sizes])
    y = torch.full((T, heads * D), 7.25, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda")
    got = gpu_lib.attention_prefill(dev16(q), batch.k, batch.v, dev(batch.table), dev(lens), dev(start), scale, gpu_lib.F32 if f32 else gpu_lib.BF16, y=y,
                                    workspace=workspace)
    assert got is y
    at = [(b, o + i) for b, (o, n) in enumerate(sizes) for i in range(n)]
    got = host(y)
    assert np.all(got[:first] == 7.25) and np.all(got[T - behind:] == 7.25)
    picked = range(len(at)) if rows is None else sorted({0, len(at) - 1} | set(int(i) for i in batch.rng.integers(0, len(at), rows)))
    check_attention(got[[first + i for i in picked]], q[[first + i for i in picked]], batch, [at[i] for i in picked], scale or D ** -0.5, f32, "D %d" % D)


@pytest.mark.parametrize("D", DIMS)
@pytest.mark.parametrize("f32", [False, True])
def test_prefill_dims(gpu_lib, D, f32):
    run_prefill(gpu_lib, [(0, 70), (33, 31), (5, 0), (63, 1), (0, 1), (-4, 6)], 4, 2, D, 32, f32, first=2, behind=3)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 3), (7, 1), (12, 1), (64, 8), (65, 1)])
@pytest.mark.parametrize("f32", [False, True])
def test_prefill_head_layouts(gpu_lib, heads, kv_heads, f32):
    run_prefill(gpu_lib, [(10, 40), (0, 129), (100, 3)], heads, kv_heads, 128, 96, f32, seed=1, rows=40)


@pytest.mark.parametrize("sizes", [[(0, 1)], [(0, 0), (3, 1)], [(0, 64)], [(0, 65)], [(0, 127), (0, 128)], [(4000, 1)], [(4000, 17)], [(0, 1030)], [(63, 1), (64, 1), (65, 2)], [(1000, 300), (1, 700)]])
@pytest.mark.parametrize("heads,kv_heads,D", [(2, 2, 128), (8, 1, 64), (4, 2, 100)])
def test_prefill_lengths(gpu_lib, sizes, heads, kv_heads, D):
    run_prefill(gpu_lib, sizes, heads, kv_heads, D, 64, len(sizes) == 1, seed=2, rows=40)


# tiles of 128 rows: a long prompt, and a chunk behind a long context, whose last tiles are filled in part
@pytest.mark.parametrize("D", [64, 100, 128, 192])
@pytest.mark.parametrize("sizes", [[(0, 2100)], [(4500, 1030)], [(0, 1500), (7, 777)]])
def test_prefill_long_runs(gpu_lib, D, sizes):
    run_prefill(gpu_lib, sizes, 64, 8, D, 64, len(sizes) == 1, seed=4, rows=24)


# rows that several workgroups share, of sequences some of which are too short for that, or end where a share begins
@pytest.mark.parametrize("D", [64, 100, 128, 256])
@pytest.mark.parametrize("sizes", [[(3000, 5)], [(2000, 20), (0, 3), (255, 1), (256, 1)], [(1500, 0), (1040, 70)], [(-2, 4), (1100, 2)]])
def test_prefill_shared_rows(gpu_lib, D, sizes):
    run_prefill(gpu_lib, sizes, 6, 2, D, 32, D != 128, seed=5, first=1, behind=2)


# weights from all alike (scores that no float of the exponent's size tells apart) to one alone
@pytest.mark.parametrize("scale,std", [(1e-39, 1.0), (1e-30, 1.0), (1e-3, 1.0), (0.7, 0.0), (1.0, 3.0), (20.0, 4.0)])
@pytest.mark.parametrize("D", [64, 128])
def test_peaked_and_flat_weights(gpu_lib, D, scale, std):
    run_prefill(gpu_lib, [(0, 300), (45, 1)], 4, 2, D, 64, True, seed=6, rows=40, scale=scale, std=std)
    run_prefill(gpu_lib, [(3000, 5)], 4, 2, D, 64, False, seed=6, scale=scale, std=std)
    run_decode(gpu_lib, [4000, 45], 4, 2, D, 64, True, seed=6, scale=scale, std=std)


def test_prefill_values_that_are_not_finite_stay_with_the_rows_that_see_them(gpu_lib):
    heads, kv_heads, D, P = 4, 2, 64, 32
    for n, at, value in [(100, 40, np.inf), (100, 99, np.nan), (300, 64, -np.inf), (70, 0, np.nan)]:
        batch = Batch([n], P, kv_heads, D, 9)
        page = batch.table[0, at // P]
        batch.cache.v[page, at % P, 0, 5] = value
        k, v = batch.cache.layout()
        q = batch.queries(n, heads, D)
        y = gpu_lib.attention_prefill(dev16(q), batch.k, dev16(v), dev(batch.table), dev([n]), dev([0, n]), y_dtype=gpu_lib.F32)
        got = host(y).reshape(n, heads, D)
        touched = np.zeros((n, heads, D), dtype=bool)
        touched[at:, : heads // kv_heads, 5] = True
        assert not np.isfinite(got[touched]).any() and np.isfinite(got[~touched]).all()
        clean = Batch([n], P, kv_heads, D, 9)
        ref = host(gpu_lib.attention_prefill(dev16(q), clean.k, clean.v, dev(clean.table), dev([n]), dev([0, n]), y_dtype=gpu_lib.F32)).reshape(n, heads, D)
        assert np.allclose(got[~touched], ref[~touched], rtol=2 ** -15, atol=2 ** -15)


def test_prefill_leaves_out_pages_that_are_not_there(gpu_lib):
    lens, sizes = [200, 150], [(100, 100), (0, 150)]
    batch = Batch(lens, 32, 2, 64, 6)
    batch.table[0, 1], batch.table[1, 0], batch.table[1, 3] = -1, 1 << 30, -2 ** 31
    q = batch.queries(250, 4, 64)
    y = gpu_lib.attention_prefill(dev16(q), batch.k, batch.v, dev(batch.table), dev(lens), dev([0, 100, 250]), y_dtype=gpu_lib.F32)
    check_attention(host(y), q, batch, [(b, o + i) for b, (o, n) in enumerate(sizes) for i in range(n)], 64 ** -0.5, True)


# ---- where they run ------------------------------------------------------------------------------------------------------------
def test_caches_beyond_32_bit_offsets(gpu_lib):
    """A cache of over 4 GiB a buffer: sequences on its last pages."""
    pages, P, H, D = 9000, 256, 8, 128
    k = torch.empty((pages, H, P // 32, D // 8, 32, 8), dtype=torch.bfloat16, device="cuda")
    v = torch.empty((pages, H, P // 32, 4, D, 8), dtype=torch.bfloat16, device="cuda")
    assert k.numel() * 2 > 1 << 32
    small = Batch([700, 300], P, H, D, 12)
    far = pages - 1 - small.table
    for b in range(2):
        for p in range(small.per):
            k[int(far[b, p])] = small.k[int(small.table[b, p])]
            v[int(far[b, p])] = small.v[int(small.table[b, p])]
    q = small.queries(2, 16, D)
    y = gpu_lib.attention_decode(dev16(q), k, v, dev(far), dev([700, 300]), y_dtype=gpu_lib.F32)
    check_attention(host(y), q, small, [(0, 699), (1, 299)], D ** -0.5, True)
    y = gpu_lib.attention_prefill(dev16(q), k, v, dev(far), dev([700, 300]), dev([0, 1, 2]), y_dtype=gpu_lib.F32)
    check_attention(host(y), q, small, [(0, 699), (1, 299)], D ** -0.5, True)
    x = small.rng.standard_normal((2, 16 + 2 * H, D)).astype(np.float32)
    for start in (None, dev([0, 1, 2])):
        k[far[0, 2]] = 0
        gpu_lib.rope_kv_append(torch.from_numpy(x.reshape(2, -1)).cuda(), None, k, v, dev(far), dev([701, 301]), 16, q_start=start)
        at = 700 % P
        got = k[int(far[0, 2]), :, at // 32, :, 16 * ((at % 32 >> 2) & 1) + 4 * (at % 32 >> 3) + (at & 3), :].reshape(H, D)
        assert np.array_equal(host(got), bf16(x[0, 16:16 + H]))


def test_strided_tables_and_another_stream(gpu_lib):
    batch = Batch([100, 65], 32, 2, 64, 13)
    wide = torch.full((2, 11), -1, dtype=torch.int32, device="cuda")
    wide[:, : batch.per] = dev(batch.table)
    q = batch.queries(2, 4, 64)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = gpu_lib.attention_decode(dev16(q), batch.k, batch.v, wide[:, : batch.per], dev([100, 65]), y_dtype=gpu_lib.F32)
    side.synchronize()
    check_attention(host(y), q, batch, [(0, 99), (1, 64)], 64 ** -0.5, True)


def test_prompt_then_tokens_in_a_graph(gpu_lib):
    """A prompt in two chunks, then tokens one by one through a captured step whose lengths grow in place: every token's attention
    is that of its definition, and the graph's replays are what eager calls give."""
    heads, kv_heads, D, P, n = 8, 2, 128, 32, 150
    rng = np.random.default_rng(21)
    B, per = 2, -(-(n + 60) // P)
    table, pages = tables(rng, B, per)
    tab = dev(table)
    freq = (10000.0 ** (-np.arange(0, D, 2) / D)).astype(np.float32)
    f = dev(freq, np.float32)
    total = [n + 12, n - 20 + 12]
    x = [bf16(rng.standard_normal((t, heads + 2 * kv_heads, D))) for t in total]
    k, v = gpu_lib.kv_cache(pages, P, kv_heads, D)
    k.fill_(float("nan")), v.fill_(float("nan"))
    out = [np.zeros((t, heads, D)) for t in total]
    queries = [np.zeros((t, heads, D)) for t in total]
    done = [0, 0]
    for chunk in ([90, 1], [n - 90, n - 21]):
        rows = np.concatenate([x[b][done[b]:done[b] + chunk[b]] for b in range(B)])
        start, lens = dev(np.cumsum([0] + chunk)), dev([done[b] + chunk[b] for b in range(B)])
        q = gpu_lib.rope_kv_append(dev16(rows.reshape(len(rows), -1)), f, k, v, tab, lens, heads, q_start=start)
        y = gpu_lib.attention_prefill(q, k, v, tab, lens, start, y_dtype=gpu_lib.F32)
        at = 0
        for b in range(B):
            out[b][done[b]:done[b] + chunk[b]] = host(y)[at:at + chunk[b]].reshape(-1, heads, D)
            queries[b][done[b]:done[b] + chunk[b]] = host(q)[at:at + chunk[b]]
            at += chunk[b]
            done[b] += chunk[b]
    lens = dev(done)
    qkv = torch.zeros((B, (heads + 2 * kv_heads) * D), dtype=torch.bfloat16, device="cuda")

    def step():
        q = gpu_lib.rope_kv_append(qkv, f, k, v, tab, lens, heads)
        return q, gpu_lib.attention_decode(q, k, v, tab, lens, y_dtype=gpu_lib.F32)

    lens.add_(1)
    qkv.copy_(dev16(np.stack([x[b][done[b]] for b in range(B)]).reshape(B, -1)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        gq, gy = step()
    for i in range(12):
        qkv.copy_(dev16(np.stack([x[b][done[b]] for b in range(B)]).reshape(B, -1)))
        graph.replay()
        eager = step()[1]
        assert torch.equal(gy, eager)
        for b in range(B):
            out[b][done[b]], queries[b][done[b]] = host(gy)[b].reshape(heads, D), host(gq)[b]
            done[b] += 1
        lens.add_(1)
    cache = Cache(pages, P, kv_heads, D)
    cache.k, cache.v = cache.from_layout(host(k), host(v))
    for b in range(B):
        keys, values, _ = cache.get(table[b], total[b])
        assert np.array_equal(values, x[b][:, heads + kv_heads:])
        for t in range(total[b]):
            o, bounds = attention(queries[b][t], keys, values, np.arange(total[b]) <= t, D ** -0.5)
            assert np.all(np.abs(out[b][t] - o) <= bounds[1]), (b, t)


def test_a_decoder_layers_attention_half(gpu_lib):
    """norm -> Q | K | V -> rotary, cache -> attention -> output projection, a ragged prompt and then a token, heads of 100: the library's own
    products in front and behind.  What the products give is the oracle's (bit for bit up to the output's bf16), what stands
    between them is held to its definition on the rows that the device computed."""
    heads, D, P = 4, 100, 32
    H = heads * D
    wqkv, wo = synth.weights(3 * H, H, config=1, layer=3), synth.weights(H, H, config=1, layer=4)
    packed, gamma = gpu_lib.quantize_weights_segmented(torch.from_numpy(wqkv).cuda(), [H, H, H])
    packed_o, gamma_o = gpu_lib.quantize_weights(torch.from_numpy(wo).cuda())
    freq = (10000.0 ** (-np.arange(0, D, 2) / D)).astype(np.float32)
    f = dev(freq, np.float32)
    rng = np.random.default_rng(33)
    table, pages = tables(rng, 2, 4)
    tab = dev(table)
    k, v = gpu_lib.kv_cache(pages, P, heads, D)
    done, keys, values = [0, 0], [np.zeros((0, heads, D))] * 2, [np.zeros((0, heads, D))] * 2
    for chunk in ([40, 70], [3, 0], [1, 1]):
        T = sum(chunk)
        x = torch.from_numpy(synth.activations(T, H, config=1, layer=T)).cuda().to(torch.bfloat16)
        lens, start = [done[b] + chunk[b] for b in range(2)], np.cumsum([0] + chunk)
        one = chunk == [1, 1]
        if one:
            qkv = gpu_lib.rmsnorm_linear_fused(x, None, 1e-6, packed, gamma, 3 * H, y_dtype=gpu_lib.BF16, segmented=True)
            q = gpu_lib.rope_kv_append(qkv, f, k, v, tab, dev(lens), heads)
            y = gpu_lib.attention_decode(q, k, v, tab, dev(lens))
            out = gpu_lib.linear_fused(y, packed_o, gamma_o, H)
        else:
            qkv = gpu_lib.linear_segmented(*gpu_lib.rmsnorm_quantize(x), packed, gamma, 3 * H, y_dtype=gpu_lib.BF16)
            q = gpu_lib.rope_kv_append(qkv, f, k, v, tab, dev(lens), heads, q_start=dev(start))
            y = gpu_lib.attention_prefill(q, k, v, tab, dev(lens), dev(start))
            out = gpu_lib.linear(*gpu_lib.quantize_acts(y), packed_o, gamma_o, H)
        rows = host(qkv).reshape(T, 3 * heads, D)
        hk, hv = Cache(pages, P, heads, D).from_layout(host(k), host(v))
        cache = Cache(pages, P, heads, D)
        cache.k, cache.v = hk, hv
        for b in range(2):
            r, pos = slice(int(start[b]), int(start[b + 1])), np.arange(done[b], lens[b])
            turned, off = rope(rows[r, : 2 * heads], pos, freq, False)
            got_k, got_v, _ = cache.get(table[b], lens[b])
            assert np.array_equal(got_v[done[b]:], rows[r, 2 * heads:])
            assert np.all(np.abs(got_k[done[b]:] - turned[:, heads:]) <= off[:, heads:] * 1.01 + BF16_HALF_STEP * np.abs(turned[:, heads:]))
            assert np.array_equal(got_k[: done[b]], keys[b]) and np.array_equal(got_v[: done[b]], values[b])      # earlier tokens stay
            qs = host(q)[r]
            assert np.all(np.abs(qs - turned[:, :heads]) <= off[:, :heads] * 1.01 + BF16_HALF_STEP * np.abs(turned[:, :heads]))
            for i in range(chunk[b]):
                o, bounds = attention(qs[i], got_k, got_v, np.arange(lens[b]) <= pos[i], D ** -0.5)
                assert np.all(np.abs(host(y)[int(start[b]) + i].reshape(heads, D) - o) <= bounds[0])
            keys[b], values[b], done[b] = got_k, got_v, lens[b]
        ref = oracle.bitlinear(y.float().cpu().numpy(), wo)
        nz = ref["y"] != 0
        assert (np.abs(host(out)[nz] - ref["y"][nz]) / np.abs(ref["y"][nz])).max() <= 1e-5


@pytest.mark.parametrize("D", [36, 256])
def test_runs_captured_without_a_call_in_front(gpu_lib, D):
    """The first launch of a head's size in the process is into a graph; its replays, with other keys and lengths in place, are eager calls'."""
    batch = Batch([1300, 90], 32, 2, D, 14)
    q, y = dev16(batch.queries(50, 4, D)), torch.zeros((50, 4 * D), dtype=torch.float32, device="cuda")
    lens, start, tab = dev([1300, 90]), dev([0, 7, 50]), dev(batch.table)
    ws = torch.empty(max(1, gpu_lib.attention_workspace(50, 4, D, batch.k, tab, prefill=True)), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        gpu_lib.attention_prefill(q, batch.k, batch.v, tab, lens, start, y_dtype=gpu_lib.F32, y=y, workspace=ws)
    for n in ([1300, 90], [700, 44], [1299, 89], [0, 43]):
        lens.copy_(dev(n))
        q.neg_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, gpu_lib.attention_prefill(q, batch.k, batch.v, tab, lens, start, y_dtype=gpu_lib.F32))
        check_attention(host(y), host(q), batch, [(0, n[0] - 7 + i) for i in range(7)] + [(1, n[1] - 43 + i) for i in range(43)], D ** -0.5, True)


def test_two_streams_with_workspaces_of_their_own(gpu_lib):
    batches = [Batch([3000, 2900], 64, 2, 128, 15), Batch([2500, 1100], 64, 2, 128, 16)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    qs = [dev16(b.queries(2, 8, 128)) for b in batches]
    tabs, lens = [dev(b.table) for b in batches], [dev(b.lens) for b in batches]
    want = [gpu_lib.attention_decode(qs[i], b.k, b.v, tabs[i], lens[i], y_dtype=gpu_lib.F32) for i, b in enumerate(batches)]
    ws = [torch.empty(gpu_lib.attention_workspace(2, 8, 128, b.k, tabs[i]), dtype=torch.uint8, device="cuda") for i, b in enumerate(batches)]
    assert all(w.numel() for w in ws)
    got = [[torch.empty_like(want[i]) for _ in range(20)] for i in range(2)]
    torch.cuda.synchronize()
    for j in range(20):
        for i, b in enumerate(batches):
            with torch.cuda.stream(streams[i]):
                gpu_lib.attention_decode(qs[i], b.k, b.v, tabs[i], lens[i], y_dtype=gpu_lib.F32, y=got[i][j], workspace=ws[i])
    torch.cuda.synchronize()
    assert all(torch.equal(got[i][j], want[i]) for i in range(2) for j in range(20))


@pytest.mark.parametrize("prefill", [False, True])
def test_with_and_without_a_workspace(gpu_lib, prefill):
    """No workspace, one that is too small, and the query's: the same values up to the order of sums."""
    lens = [1500, 800]
    batch = Batch(lens, 64, 2, 128, 17)
    q = batch.queries(2, 8, 128)
    tab = dev(batch.table)
    need = gpu_lib.attention_workspace(2, 8, 128, batch.k, tab, prefill=prefill)
    assert need > 0
    for n in (0, need - 16, need, need + 48):
        ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
        if prefill:
            y = gpu_lib.attention_prefill(dev16(q), batch.k, batch.v, tab, dev(lens), dev([0, 1, 2]), y_dtype=gpu_lib.F32, workspace=ws)
        else:
            y = gpu_lib.attention_decode(dev16(q), batch.k, batch.v, tab, dev(lens), y_dtype=gpu_lib.F32, workspace=ws)
        check_attention(host(y), q, batch, [(0, 1499), (1, 799)], 128 ** -0.5, True, "%d of %d bytes" % (n, need))


def test_refusals_of_the_binding(gpu_lib):
    batch = Batch([40, 33], 32, 2, 64, 18)
    tab, lens, q = dev(batch.table), dev([40, 33]), dev16(batch.queries(2, 4, 64))
    start = dev([0, 1, 2])
    ok = dict(q=q, k_cache=batch.k, v_cache=batch.v, page_table=tab, kv_len=lens)
    gpu_lib.attention_decode(**ok)
    wrong = [("q", q.float(), TypeError), ("q", q[0], ValueError), ("q", q[:1], ValueError), ("q", q.transpose(0, 1), ValueError), ("q", q[:, :3].contiguous(), gpu_lib.BitnetError),
             ("q", q[..., :32].contiguous(), ValueError), ("k_cache", batch.k.float(), TypeError), ("k_cache", batch.k[0], ValueError), ("v_cache", batch.v[:-1], ValueError),
             ("v_cache", batch.k, ValueError), ("page_table", tab.long(), TypeError), ("page_table", tab.t(), ValueError), ("page_table", tab[0], ValueError),
             ("kv_len", lens[:1], ValueError), ("kv_len", lens.long(), TypeError), ("scale", 0.0, gpu_lib.BitnetError), ("scale", float("nan"), gpu_lib.BitnetError),
             ("y_dtype", gpu_lib.I32, ValueError), ("y_dtype", 9, KeyError), ("y", torch.empty((2, 255), dtype=torch.bfloat16, device="cuda"), ValueError),
             ("y", torch.empty((2, 256), dtype=torch.float32, device="cuda"), TypeError)]
    for name, value, error in wrong:
        for call, more in ((gpu_lib.attention_decode, {}), (gpu_lib.attention_prefill, {"q_start": start})):
            if call is gpu_lib.attention_prefill and name == "q" and value.dim() == 3 and value.shape[0] == 1:
                continue                                     # one row for two sequences is a batch of runs like any other
            with pytest.raises(error):
                call(**{**ok, **more, name: value})
    for bad, error in ((start[:2], ValueError), (start.long(), TypeError), (None, gpu_lib.BitnetError)):
        with pytest.raises(error):
            gpu_lib.attention_prefill(**ok, q_start=bad)
    qkv, f = torch.zeros((2, 8 * 64), device="cuda"), torch.ones(32, device="cuda")
    args = dict(qkv=qkv, inv_freq=f, k_cache=batch.k, v_cache=batch.v, page_table=tab, kv_len=lens, heads=4)
    gpu_lib.rope_kv_append(**args)
    for name, value, error in [("qkv", qkv.half(), TypeError), ("qkv", qkv[0], ValueError), ("qkv", qkv[:, :500].contiguous(), ValueError), ("qkv", qkv[:1], gpu_lib.BitnetError),
                               ("heads", 3, ValueError), ("heads", 0, ValueError), ("heads", -4, ValueError), ("inv_freq", f.double(), TypeError), ("inv_freq", f[None], ValueError),
                               ("inv_freq", torch.ones(33, device="cuda"), gpu_lib.BitnetError), ("q", torch.empty((2, 4, 63), dtype=torch.bfloat16, device="cuda"), ValueError),
                               ("q_start", start[:2], ValueError)]:
        with pytest.raises(error):
            gpu_lib.rope_kv_append(**{**args, name: value})
    for bad in ((0, 32, 1, 64), (4, 40, 1, 64), (4, 32, 1, 63), (4, 32, 1, 258)):
        with pytest.raises(gpu_lib.BitnetError):
            gpu_lib.kv_cache(*bad)
