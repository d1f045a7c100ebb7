"""The cache's operators of a serving loop as they are used: one behind another, captured and replayed, on streams of their own, with workspaces of exactly the
bytes that were asked for, on caches beyond 32-bit offsets, at the ends of their ranges, beside values that are not finite."""
import numpy as np
import pytest

from attention_ref import BF16_HALF_STEP, F32_HALF_STEP, Cache, attention, bf16
from cache_ref import evict, norm_rope, weights
from test_gpu_attention import Batch, check_attention, dev, dev16, host, tables
from test_gpu_cache_ops import Shared, run_evict, run_norm_append, run_shared, run_weights

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def captured(step):
    """A graph of `step`, run once on a side stream in front, and what it returned under capture."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    return graph, out


def test_a_serving_loop_that_evicts(gpu_lib):
    """A prompt, normed, turned and weighed; eviction; tokens through a captured step with shifted positions; eviction again; tokens.  Every stage is held to
    its definition on what the device had in front of it."""
    heads, kv_heads, D, P, B, keep, recent = 8, 2, 64, 32, 2, 50, 12
    rng = np.random.default_rng(71)
    prompt, per = [120, 45], 5
    numbers = rng.permutation(40).astype(np.int32)
    rows = [numbers[: B * per].reshape(B, per), numbers[B * per: 2 * B * per].reshape(B, per)]
    freq = (10000.0 ** (-np.arange(0, D, 2) / D)).astype(np.float32)
    qg, kg = ((1 + 0.2 * rng.standard_normal(D)).astype(np.float32) for _ in range(2))
    f, qgd, kgd = dev(freq, np.float32), dev(qg, np.float32), dev(kg, np.float32)
    k, v = gpu_lib.kv_cache(40, P, kv_heads, D)
    k.fill_(float("nan")), v.fill_(float("nan"))
    table, lens, shift = dev(rows[0]), dev(prompt), torch.zeros(B, dtype=torch.int32, device="cuda")
    acc = torch.full((B, kv_heads, per * P), float("nan"), device="cuda")
    x = [bf16(rng.standard_normal((n, heads + 2 * kv_heads, D)) * 2) for n in prompt]
    start = dev(np.cumsum([0] + prompt))
    qkv = dev16(np.concatenate(x).reshape(sum(prompt), -1))
    q = gpu_lib.norm_rope_kv_append(qkv, f, k, v, table, lens, heads, qgd, kgd, q_start=start, shift=shift)
    y = gpu_lib.attention_prefill_weights(q, k, v, table, lens, start, acc, y_dtype=gpu_lib.F32)

    def whole(row, n):
        c = Cache(40, P, kv_heads, D)
        c.k, c.v = c.from_layout(host(k), host(v))
        return c.get(row, n)[:2]

    model = []                                               # of each sequence the accumulators in 64 bits and their bounds
    at = np.concatenate([[0], np.cumsum(prompt)])
    for b, n in enumerate(prompt):
        keys, values = whole(rows[0][b], n)
        want, off = norm_rope(x[b][:, heads:heads + kv_heads], np.arange(n), freq, False, kg, 1e-6, True)
        assert np.all(np.abs(keys - want) <= off * 1.01 + BF16_HALF_STEP * np.abs(want)) and np.array_equal(values, x[b][:, heads + kv_heads:])
        w, e = np.zeros((kv_heads, n)), np.zeros((kv_heads, n))
        for i in range(n):
            o, bounds = attention(host(q)[at[b] + i], keys, values, np.arange(n) <= i, D ** -0.5)
            assert np.all(np.abs(host(y)[at[b] + i].reshape(heads, D) - o) <= bounds[1])
            one, more = weights(host(q)[at[b] + i], keys, np.arange(n) <= i, D ** -0.5)
            w, e = w + one, e + more
        e += (n * heads // kv_heads + 2) * F32_HALF_STEP * w
        assert np.all(np.abs(host(acc)[b, :, :n] - w) <= e)
    one = torch.zeros((B, (heads + 2 * kv_heads) * D), dtype=torch.bfloat16, device="cuda")
    gone = np.zeros(B, dtype=np.int64)
    for turn in range(2):
        before, had = lens.cpu().numpy(), host(acc)
        old = [whole(rows[turn][b], before[b]) for b in range(B)]
        table = dev(rows[1 - turn])
        new_len, acc, kept = gpu_lib.kv_evict(k, v, dev(rows[turn]), lens, acc, keep, recent, table)
        for b in range(B):
            keys, values = whole(rows[1 - turn][b], int(new_len[b]))
            for h in range(kv_heads):
                stay = evict(had[b, h].astype(np.float32), before[b], keep, recent)
                assert kept[b, h, : len(stay)].tolist() == stay and len(stay) == int(new_len[b])
                assert np.array_equal(keys[:, h], old[b][0][stay, h]) and np.array_equal(values[:, h], old[b][1][stay, h])
                assert np.array_equal(host(acc)[b, h, : len(stay)], had[b, h, stay])
        gone += before - new_len.cpu().numpy()
        shift, lens = dev(gone), new_len.clone()

        def step():
            q = gpu_lib.norm_rope_kv_append(one, f, k, v, table, lens, heads, qgd, kgd, shift=shift)
            return q, gpu_lib.attention_decode_weights(q, k, v, table, lens, acc, y_dtype=gpu_lib.F32)

        saved = acc.clone()
        lens.add_(1)
        graph, (gq, gy) = captured(step)
        acc.copy_(saved)
        for i in range(9):
            xs = bf16(rng.standard_normal((B, heads + 2 * kv_heads, D)) * 2)
            one.copy_(dev16(xs.reshape(B, -1)))
            had = acc.clone()
            graph.replay()
            after = acc.clone()
            acc.copy_(had)
            assert torch.equal(gy, step()[1])
            for b in range(B):                               # behind a sequence's tokens there is whatever memory held
                assert torch.equal(acc[b, :, : int(lens[b])], after[b, :, : int(lens[b])])
            for b in range(B):
                n = int(lens[b])
                keys, values = whole(rows[1 - turn][b], n)
                for part, gain, got in ((slice(0, heads), qg, host(gq)[b][None]), (slice(heads, heads + kv_heads), kg, keys[n - 1][None])):
                    want, off = norm_rope(xs[b][None, part], np.array([n - 1 + gone[b]]), freq, False, gain, 1e-6, True)
                    assert np.all(np.abs(got - want) <= off * 1.01 + BF16_HALF_STEP * np.abs(want))
                o, bounds = attention(host(gq)[b], keys, values, np.ones(n, dtype=bool), D ** -0.5)
                assert np.all(np.abs(host(gy)[b].reshape(heads, D) - o) <= bounds[1])
                w, e = weights(host(gq)[b], keys, np.ones(n, dtype=bool), D ** -0.5)
                was = host(had)[b, :, :n]
                was[:, n - 1] = 0
                assert np.all(np.abs(host(acc)[b, :, :n] - was - w) <= e + 4 * F32_HALF_STEP * (was + w))
            lens.add_(1)
        lens.sub_(1)


def test_prefixes_in_graphs_that_share_a_workspace(gpu_lib):
    """Two captured calls on one workspace, one behind the other, with lengths, prefixes and queries that change in place, eager calls between."""
    batch = Shared([400, 350, 333, 90], [3, 1], [300, 64], 32, 2, 100, 81)
    table, lens, start, prefix = dev(batch.table), dev(batch.lens), dev(batch.start), dev(batch.prefix)
    q = dev16(batch.queries(4, 6, 100))
    need = gpu_lib.attention_shared_workspace(2, 6, 100, batch.k, table, gpu_lib.F32)
    ws, y = torch.empty(need, dtype=torch.uint8, device="cuda"), [torch.zeros((4, 600), device="cuda") for _ in range(2)]
    qs = [q, (-q).contiguous()]
    graphs = [captured(lambda i=i: gpu_lib.attention_decode_shared(qs[i], batch.k, batch.v, table, lens, start, prefix, y_dtype=gpu_lib.F32, y=y[i], workspace=ws))[0] for i in range(2)]
    for n, p in (([400, 350, 333, 90], [300, 64]), ([301, 300, 299, 64], [300, 64]), ([400, 350, 333, 90], [12, 0]), ([0, 1, 0, 0], [300, 64]), ([400, 350, 333, 90], [300, 64])):
        lens.copy_(dev(n)), prefix.copy_(dev(p))
        if p == [12, 0]:                                     # the other sequences' own pages hold nothing there: the first one's row alone
            lens[1:] = 0
        for i in range(2):
            graphs[i].replay()
        got = [t.clone() for t in y]
        for i in range(2):
            assert torch.equal(got[i], gpu_lib.attention_decode_shared(qs[i], batch.k, batch.v, table, lens, start, prefix, y_dtype=gpu_lib.F32))
            assert torch.isfinite(got[i]).all()


def test_eviction_and_weights_in_graphs(gpu_lib):
    batch = Batch([300, 170], 32, 2, 64, 82, per=10)
    k, v = torch.cat([batch.k, torch.zeros_like(batch.k[:8])]), torch.cat([batch.v, torch.zeros_like(batch.v[:8])])
    pages = batch.k.shape[0]
    table, out, lens, start = dev(batch.table), dev(np.arange(pages, pages + 8).reshape(2, 4)), dev([300, 170]), dev([0, 40, 50])
    q, acc = dev16(batch.queries(50, 4, 64)), torch.rand((2, 2, 320), device="cuda")
    w_out, len_out, kept = torch.zeros((2, 2, 128), device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros((2, 2, 100), dtype=torch.int32, device="cuda")

    def step():
        y = gpu_lib.attention_prefill_weights(q, k, v, table, lens, start, acc)
        gpu_lib.kv_evict(k, v, table, lens, acc, 100, 30, out, kv_len_out=len_out, weights_out=w_out, kept=kept)
        return y

    graph, y = captured(step)
    for n in ([300, 170], [120, 10], [44, 170], [300, 169]):
        lens.copy_(dev(n))
        for _ in range(2):
            q.neg_()
            had = acc.clone()
            graph.replay()
            got = [t.clone() for t in (y, acc, len_out, w_out, kept, k, v)]
            acc.copy_(had)
            again = step()
            assert all(torch.equal(a, b) for a, b in zip(got[1:5], (acc, len_out, w_out, kept))) and torch.equal(got[0], again)
            assert torch.equal(got[5].view(torch.int16), k.view(torch.int16)) and torch.equal(got[6].view(torch.int16), v.view(torch.int16))


@pytest.mark.parametrize("B,heads,kv_heads,D,cap", [(1, 8, 8, 64, 4096), (5, 16, 2, 100, 2080), (40, 8, 1, 128, 1024), (3, 6, 2, 250, 320)])
def test_workspaces_are_not_left(gpu_lib, B, heads, kv_heads, D, cap):
    """Scratch of exactly the bytes of the query, full of NaN, in the middle of a buffer whose other bytes stay."""
    lens = [cap - 7 * b for b in range(B)]
    batch = Batch(lens, 32, kv_heads, D, 83)
    q, tab, n = batch.queries(B, heads, D), dev(batch.table), dev(lens)
    start, prefix = dev([0, B]), dev([cap // 2])
    tab[:, : cap // 2 // 32] = tab[:1, : cap // 2 // 32]
    runs = dev(np.arange(B + 1))
    for y_dtype in (gpu_lib.F32, gpu_lib.BF16):
        calls = [(gpu_lib.attention_shared_workspace(1, heads, D, batch.k, tab, y_dtype),
                  lambda ws: [gpu_lib.attention_decode_shared(dev16(q), batch.k, batch.v, tab, n, start, prefix, y_dtype=y_dtype, workspace=ws)])]
        for prefill in (False, True):
            def weighed(ws, prefill=prefill):
                acc = torch.ones((B, kv_heads, batch.per * 32), device="cuda")
                if prefill:
                    return [gpu_lib.attention_prefill_weights(dev16(q), batch.k, batch.v, tab, n, runs, acc, y_dtype=y_dtype, workspace=ws), acc]
                return [gpu_lib.attention_decode_weights(dev16(q), batch.k, batch.v, tab, n, acc, y_dtype=y_dtype, workspace=ws), acc]
            calls.append((gpu_lib.attention_weights_workspace(B, heads, D, batch.k, tab, prefill, y_dtype), weighed))
        for need, call in calls:
            room = torch.full((need + 8192,), 0xFF, dtype=torch.uint8, device="cuda")
            got, want = call(room[4096: 4096 + need]), call(None)
            assert all(torch.equal(a, b) and torch.isfinite(a).all() for a, b in zip(got, want))
            assert (room[:4096] == 0xFF).all() and (room[4096 + need:] == 0xFF).all()
            with pytest.raises(gpu_lib.BitnetError):
                call(room[: need - 16])


def test_on_streams_of_their_own(gpu_lib):
    batches = [Shared([900, 950, 1200], [3], [800], 64, 2, 128, 84), Shared([500, 700, 640], [3], [450], 64, 2, 128, 85)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    args = [(dev16(b.queries(3, 8, 128)), b.k, b.v, dev(b.table), dev(b.lens)) for b in batches]
    more = [(dev(b.start), dev(b.prefix)) for b in batches]
    accs = [torch.zeros((3, 2, b.per * 64), device="cuda") for b in batches]
    tabs = [a[3].clone() for a in args]
    for t, b in zip(tabs, batches):                          # every row whole, for the calls that know of no prefixes
        t[:, : int(b.prefix[0]) // 64] = t[:1, : int(b.prefix[0]) // 64]
    lens = [dev([int(b.prefix[0]) // 64 * 64] * 3) for b in batches]
    want = [gpu_lib.attention_decode_shared(*a, *m) for a, m in zip(args, more)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(12):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(gpu_lib.attention_decode_shared(*args[i], *more[i]))
                gpu_lib.attention_decode_weights(*args[i][:3], tabs[i], lens[i], accs[i])
    torch.cuda.synchronize()
    assert all(torch.equal(g, want[i]) for i in range(2) for g in got[i])
    for i in range(2):
        one = torch.zeros_like(accs[i])
        gpu_lib.attention_decode_weights(*args[i][:3], tabs[i], lens[i], one)
        n = int(lens[i][0])
        assert torch.allclose(accs[i][:, :, : n - 1], 12 * one[:, :, : n - 1], rtol=13 * 2 ** -24, atol=0) and torch.equal(accs[i][:, :, n - 1], one[:, :, n - 1])


def test_caches_beyond_32_bit_offsets(gpu_lib):
    """A cache of over 4 GiB a buffer: sequences, and what stays of them, on its last pages."""
    pages, P, H, D = 9000, 256, 8, 128
    k = torch.empty((pages, H, P // 32, D // 8, 32, 8), dtype=torch.bfloat16, device="cuda")
    v = torch.empty((pages, H, P // 32, 4, D, 8), dtype=torch.bfloat16, device="cuda")
    small = Shared([700, 600], [2], [520], P, H, D, 86)
    far = pages - 1 - small.table
    for b in range(2):
        for p in range(small.per):
            k[int(far[b, p])], v[int(far[b, p])] = small.k[int(small.table[b, p])], small.v[int(small.table[b, p])]
    q = small.queries(2, 16, D)
    lens, tab = dev([700, 600]), dev(far)
    y = gpu_lib.attention_decode_shared(dev16(q), k, v, tab, lens, dev([0, 2]), dev([520]), y_dtype=gpu_lib.F32)
    near = gpu_lib.attention_decode_shared(dev16(q), small.k, small.v, dev(small.table), lens, dev([0, 2]), dev([520]), y_dtype=gpu_lib.F32)
    assert torch.equal(y, near) and torch.isfinite(y).all()
    one, acc = dev(far[:1]), [torch.ones((1, H, 768), device="cuda") for _ in range(4)]
    n, start = lens[:1].clone(), dev([0, 1])
    for i, (a, b, t) in enumerate(((k, v, one), (small.k, small.v, dev(small.table[:1])))):
        gpu_lib.attention_decode_weights(dev16(q[:1]), a, b, t, n, acc[i], y_dtype=gpu_lib.F32)
        gpu_lib.attention_prefill_weights(dev16(q[:1]), a, b, t, n, start, acc[2 + i], y_dtype=gpu_lib.F32)
    assert torch.equal(acc[0], acc[1]) and torch.equal(acc[2], acc[3])
    to = dev([[pages - 40, 5]])
    _, _, kept = gpu_lib.kv_evict(k, v, one, n, acc[0], 300, 100, to)
    t, at = torch.arange(300, device="cuda"), kept[0].long()
    for cache, values in ((k, False), (v, True)):
        def tokens(page, pos, h):
            j = pos % P
            if values:
                return cache.permute(0, 1, 2, 3, 5, 4)[page, h, j // 32, j % 32 // 8, j % 8]
            return cache[page, h, j // 32, :, 16 * (j // 4 % 2) + 4 * (j % 32 // 8) + j % 4].reshape(len(pos), -1)
        for h in (0, H - 1):
            assert torch.equal(tokens(to[0].long()[t // P], t, h), tokens(one[0].long()[at[h] // P], at[h], h))


def test_strided_tables_and_odd_addresses(gpu_lib):
    """Tables with rows of their own stride, queries at an odd multiple of two bytes, outputs and accumulators at their element's alignment."""
    batch = Shared([100, 65, 80], [3], [50], 32, 2, 90, 87)
    wide = torch.full((3, 11), -1, dtype=torch.int32, device="cuda")
    wide[:, : batch.per] = dev(batch.table)
    q = dev16(batch.queries(3, 4, 90))
    odd = torch.zeros(q.numel() + 1, dtype=torch.bfloat16, device="cuda")[1:].view(q.shape)
    odd.copy_(q)
    lens, start, prefix = dev(batch.lens), dev(batch.start), dev(batch.prefix)
    y = torch.zeros(3 * 360 + 1, dtype=torch.bfloat16, device="cuda")[1:].view(3, 360)
    got = gpu_lib.attention_decode_shared(odd, batch.k, batch.v, wide[:, : batch.per], lens, start, prefix, y=y)
    assert got is y and torch.equal(y, gpu_lib.attention_decode_shared(q, batch.k, batch.v, dev(batch.table), lens, start, prefix))
    one, runs = dev([50]), dev([0, 3])
    for prefill in (False, True):
        accs = [torch.full((2 * 128 + 1,), 2.0, device="cuda")[1:].view(1, 2, 128), torch.full((1, 2, 128), 2.0, device="cuda")]
        for acc, qq, tab in ((accs[0], odd, wide[:1, : batch.per]), (accs[1], q, dev(batch.table)[:1])):
            if prefill:
                gpu_lib.attention_prefill_weights(qq, batch.k, batch.v, tab, one, runs, acc)
            else:
                gpu_lib.attention_decode_weights(qq[:1], batch.k, batch.v, tab, one, acc)
        assert torch.equal(*accs) and torch.isfinite(accs[0]).all()


@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("D", [24, 100, 128, 192])
@pytest.mark.parametrize("f32", [False, True])
def test_values_that_are_not_finite(gpu_lib, value, D, f32):
    """One among a prefix's values, one among a sequence's own: NaN in the dim of the rows that see it, and all else as without them."""
    heads, kv_heads, t = 4, 2, gpu_lib.F32 if f32 else gpu_lib.BF16
    for counts, lens, prefix in (([3], [150, 90, 260], 85), ([50], [150, 40, 260] + [100] * 47, 85), ([3], [40, 150, 260], 85)):
        for at, owner in ((70, 0), (84, 0), (100, 2)):
            batch = Shared(lens, counts, [prefix], 32, kv_heads, D, 88)
            args = (batch.k, dev(batch.table), dev(lens), dev(batch.start), dev(batch.prefix))
            q = dev16(batch.queries(len(lens), heads, D))
            batch.cache.v[batch.table[owner, at // 32], at % 32, 0, 1] = value
            marked = dev16(batch.cache.layout()[1])
            y, want = (host(gpu_lib.attention_decode_shared(q, args[0], v, *args[1:], y_dtype=t)).reshape(-1, heads, D) for v in (marked, batch.v))
            touched = np.zeros(y.shape, dtype=bool)
            for b, n in enumerate(lens):
                if n > at and (at < prefix or b == owner):
                    touched[b, : heads // kv_heads, 1] = True
            assert np.isnan(y[touched]).all() and np.array_equal(y[~touched], want[~touched]) and np.isfinite(want).all()


def test_what_is_not_finite_behind_a_row_reaches_no_weight(gpu_lib):
    """Caches whose unused places are infinite, queries of other sequences that are NaN: a sequence's weights are its own."""
    batch = Batch([70, 90], 32, 2, 64, 89, per=4)
    k, v = batch.cache.layout()
    for fill in (np.inf, -np.inf):
        kk, vv = dev16(np.where(np.isnan(k), fill, k)), dev16(np.where(np.isnan(v), fill, v))
        q = batch.queries(12, 4, 64)
        q[5:] = np.nan
        accs = []
        for cache in ((batch.k, batch.v), (kk, vv)):
            acc = torch.ones((2, 2, 128), device="cuda")
            y = gpu_lib.attention_prefill_weights(dev16(q), *cache, dev(batch.table), dev([70, 90]), dev([0, 5, 12]), acc, scale=3.0, y_dtype=gpu_lib.F32)
            accs.append((acc[0].clone(), y[:5].clone(), acc[1, :, 90:].clone()))
        assert all(torch.equal(a, b) for a, b in zip(*accs)) and torch.isfinite(accs[0][0]).all() and torch.isfinite(accs[0][1]).all()


@pytest.mark.parametrize("kv_heads,D", [(1, 64), (4, 100), (16384, 2)])
def test_16384_heads(gpu_lib, kv_heads, D):
    heads = 16384
    run_norm_append(gpu_lib, [(30, 1), (64, 1)], heads, kv_heads, D, 32, False, False, one=True)
    run_norm_append(gpu_lib, [(30, 3), (0, 1)], heads, kv_heads, D, 32, False, True)
    run_shared(gpu_lib, [40, 33], [2], [32], heads, kv_heads, D, 32, False, seed=61)
    run_weights(gpu_lib, [(39, 1), (0, 1)], heads, kv_heads, D, 32, True, True, seed=62)
    run_weights(gpu_lib, [(30, 3), (0, 1)], heads, kv_heads, D, 32, False, False, seed=63)


def test_very_many_sequences(gpu_lib):
    """100000 sequences of one token or two, in groups of one, two or none; many of them in one group."""
    B, heads, D = 100000, 4, 8
    k, v = gpu_lib.kv_cache(B, 32, 2, D)
    g = torch.Generator(device="cuda").manual_seed(3)
    k.normal_(generator=g), v.normal_(generator=g)
    table = torch.arange(B, device="cuda", dtype=torch.int32).view(B, 1)
    lens = torch.randint(0, 3, (B,), device="cuda", generator=g, dtype=torch.int32)
    q = torch.randn((B, heads, D), device="cuda", generator=g, dtype=torch.float32).to(torch.bfloat16)
    want = gpu_lib.attention_decode(q, k, v, table, lens, y_dtype=gpu_lib.F32)
    start = torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), torch.randint(0, 3, (50000,), device="cuda", generator=g, dtype=torch.int32).cumsum(0).to(torch.int32)])
    none = torch.zeros(50000, dtype=torch.int32, device="cuda")
    got = gpu_lib.attention_decode_shared(q, k, v, table, lens, start.clamp_(max=B), none, y_dtype=gpu_lib.F32)
    assert torch.allclose(got, want, rtol=1e-5, atol=1e-6)
    acc = torch.full((B, 2, 32), 3.0, device="cuda")
    got = gpu_lib.attention_decode_weights(q, k, v, table, lens, acc, y_dtype=gpu_lib.F32)
    assert torch.allclose(got, want, rtol=1e-5, atol=1e-6)
    held = torch.arange(32, device="cuda") < lens[:, None]
    total = torch.where(held[:, None], acc, torch.zeros_like(acc)).sum(-1)
    assert torch.allclose(total, torch.where(lens > 0, 2.0 + 3.0 * (lens - 1), 0.0)[:, None].expand_as(total), rtol=1e-5) and (acc[~held[:, None].expand_as(acc)] == 3.0).all()
    same = torch.zeros_like(table)                           # all on one page, all in one group
    full = torch.full_like(lens, 2)
    got = gpu_lib.attention_decode_shared(q, k, v, same, full, dev([0, B]), dev([2]), y_dtype=gpu_lib.F32)
    assert torch.allclose(got, gpu_lib.attention_decode(q, k, v, same, full, y_dtype=gpu_lib.F32), rtol=1e-5, atol=1e-6)


def test_a_hundred_thousand_tokens(gpu_lib):
    """Beyond what the choice of an eviction holds in registers, and many splits of a row."""
    run_evict(gpu_lib, [100000, 70001], 1, 2, 256, 30000, 5, kind="ties", seed=9)
    run_evict(gpu_lib, [100000], 1, 2, 256, 3, 0, kind="signs", seed=9, in_place=True)
    run_shared(gpu_lib, [100000, 90001], [2], [90000], 4, 2, 24, 256, True, seed=9)
    run_weights(gpu_lib, [(99999, 1), (8, 1)], 4, 2, 24, 256, True, True, seed=9)
    run_weights(gpu_lib, [(99990, 3), (8, 1)], 4, 2, 24, 256, True, False, seed=9)


def test_refusals_of_the_binding(gpu_lib):
    batch = Batch([40, 33], 32, 2, 64, 18)
    tab, lens, q = dev(batch.table), dev([40, 33]), dev16(batch.queries(2, 4, 64))
    start, acc = dev([0, 1, 2]), torch.zeros((2, 2, 64), device="cuda")
    ok = dict(q=q, k_cache=batch.k, v_cache=batch.v, page_table=tab, kv_len=lens)
    calls = [(gpu_lib.attention_decode_shared, dict(prefix_start=dev([0, 2]), prefix_len=dev([10]))), (gpu_lib.attention_decode_weights, dict(weights=acc)),
             (gpu_lib.attention_prefill_weights, dict(q_start=start, weights=acc))]
    wrong = [("q", q.float(), TypeError), ("q", q[0], ValueError), ("q", q.transpose(0, 1), ValueError), ("q", q[:, :3].contiguous(), gpu_lib.BitnetError),
             ("q", q[..., :32].contiguous(), ValueError), ("k_cache", batch.k.float(), TypeError), ("v_cache", batch.v[:-1], ValueError), ("page_table", tab.long(), TypeError),
             ("page_table", tab[0], ValueError), ("kv_len", lens[:1], ValueError), ("scale", 0.0, gpu_lib.BitnetError), ("y_dtype", gpu_lib.I32, ValueError),
             ("y", torch.empty((2, 255), dtype=torch.bfloat16, device="cuda"), ValueError), ("workspace", torch.empty(16, dtype=torch.uint8, device="cuda"), gpu_lib.BitnetError),
             ("workspace", torch.empty(0, dtype=torch.uint8, device="cuda"), gpu_lib.BitnetError), ("workspace", torch.empty(1 << 20, dtype=torch.uint8), TypeError)]
    for call, more in calls:
        call(**ok, **more)
        for name, value, error in wrong:
            with pytest.raises(error):
                call(**{**ok, **more, name: value})
        for name, bads in dict(weights=[(acc.double(), TypeError), (acc[0], ValueError), (acc[:, :1], ValueError), (acc[:1], ValueError), (acc[:, :, :63].contiguous(), gpu_lib.BitnetError),
                                        (acc.transpose(1, 2), ValueError)],
                               q_start=[(start[:2], ValueError), (start.long(), TypeError), (None, TypeError)],
                               prefix_start=[(dev([0, 1, 2]), ValueError), (dev([0, 2]).long(), TypeError), (None, TypeError)],
                               prefix_len=[(dev([[10]]), ValueError), (dev([10]).float(), TypeError), (dev([]), gpu_lib.BitnetError)]).items():
            for value, error in bads if name in more else []:
                with pytest.raises(error):
                    call(**{**ok, **more, name: value, **(dict(prefix_start=dev([0])) if name == "prefix_len" and value.numel() == 0 else {})})
    with pytest.raises(ValueError):
        gpu_lib.attention_decode_weights(**{**ok, "q": q[:1]}, weights=acc)
    out = dev([[0], [1]])
    args = dict(k_cache=batch.k, v_cache=batch.v, page_table=tab, kv_len=lens, weights=acc, keep=20, recent=5, page_table_out=out)
    bad_out = torch.zeros((2, 2, 19), device="cuda")
    for name, value, error in [("k_cache", batch.k.float(), TypeError), ("k_cache", batch.k[0], ValueError), ("v_cache", batch.v[:-1], ValueError), ("weights", acc[0], ValueError),
                               ("weights", acc[:, :, :63].contiguous(), gpu_lib.BitnetError), ("keep", 0, ValueError), ("keep", 33, ValueError), ("keep", -1, ValueError),
                               ("recent", -1, gpu_lib.BitnetError), ("recent", 21, gpu_lib.BitnetError), ("page_table_out", out[:1], ValueError), ("page_table_out", out.long(), TypeError),
                               ("page_table_out", out[0], ValueError), ("page_table_out", None, TypeError), ("kv_len_out", lens[:1], ValueError), ("kv_len_out", lens.long(), TypeError),
                               ("weights_out", bad_out, gpu_lib.BitnetError), ("kept", torch.zeros((2, 2, 19), dtype=torch.int32, device="cuda"), ValueError)]:
        with pytest.raises(error):
            gpu_lib.kv_evict(**{**args, name: value})
    qkv, f, gain = torch.zeros((2, 8 * 64), device="cuda"), torch.ones(32, device="cuda"), torch.ones(64, device="cuda")
    args = dict(qkv=qkv, inv_freq=f, k_cache=batch.k, v_cache=batch.v, page_table=tab, kv_len=lens, heads=4, q_gain=gain, k_gain=gain)
    gpu_lib.norm_rope_kv_append(**args)
    for name, value, error in [("qkv", qkv.half(), TypeError), ("qkv", qkv[:, :500].contiguous(), ValueError), ("qkv", qkv[:1], gpu_lib.BitnetError), ("heads", 3, ValueError),
                               ("inv_freq", f.double(), TypeError), ("q_gain", gain[:63].contiguous(), ValueError), ("k_gain", gain.double(), TypeError), ("q_gain", gain[None], ValueError),
                               ("eps", -1.0, gpu_lib.BitnetError), ("eps", float("nan"), gpu_lib.BitnetError), ("shift", lens[:1], ValueError), ("shift", lens.long(), TypeError),
                               ("q", torch.empty((2, 4, 63), dtype=torch.bfloat16, device="cuda"), ValueError), ("q_start", start[:2], ValueError)]:
        with pytest.raises(error):
            gpu_lib.norm_rope_kv_append(**{**args, name: value})
