"""The attention half at the ends of its documented ranges: 16384 heads, four million rows, a hundred thousand sequences, positions up to 2^31."""
import numpy as np
import pytest

from attention_ref import BF16_HALF_STEP, F32_HALF_STEP, bf16
from test_gpu_attention import dev, dev16, host, run_append, run_decode, run_prefill

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("kv_heads,D", [(1, 64), (4, 100), (16384, 2)])
def test_16384_heads(gpu_lib, kv_heads, D):
    heads = 16384
    run_append(gpu_lib, [(30, 1), (64, 1)], heads, kv_heads, D, 32, False, False, one=True)
    run_append(gpu_lib, [(30, 3), (0, 1)], heads, kv_heads, D, 32, False, True)
    run_decode(gpu_lib, [40, 1], heads, kv_heads, D, 32, False, seed=61)
    run_prefill(gpu_lib, [(30, 3), (0, 1)], heads, kv_heads, D, 32, False, seed=62)


def whole(x, kv_heads, D, values):
    """A cache buffer of pages of 32 tokens -> [pages, kv heads, 32, D] fp64 on the device."""
    t = torch.arange(32, device="cuda")
    if values:
        return x[:, :, 0].permute(0, 1, 2, 4, 3).reshape(x.shape[0], kv_heads, 32, -1)[..., :D].double()
    return x[:, :, 0].permute(0, 1, 3, 2, 4)[:, :, 16 * (t // 4 % 2) + 4 * (t // 8) + t % 4].reshape(x.shape[0], kv_heads, 32, -1)[..., :D].double()


def causal(q, k, v, scale):
    """q, k, v [B, n, D] fp64, D small -> (o, the bound of an fp32 result), elementwise (attention_ref has the derivation)."""
    s = (q[:, :, None] * k[:, None]).sum(-1) * scale
    size = (q[:, :, None] * k[:, None]).abs().sum(-1).amax(-1) * scale
    n, m = q.shape[1], k.shape[1]
    s.masked_fill_(torch.arange(m, device="cuda")[None] > torch.arange(m - n, m, device="cuda")[:, None], -float("inf"))
    p = torch.softmax(s, dim=-1)
    o, weight = (p[..., None] * v[:, None]).sum(2), (p[..., None] * v[:, None].abs()).sum(2)
    return o, weight * ((2 * (q.shape[2] + 8) * size + 2 * m + 64) * F32_HALF_STEP + BF16_HALF_STEP ** 2)[..., None] * 1.01 + F32_HALF_STEP * o.abs() + 1e-37


def test_four_million_rows_of_many_sequences(gpu_lib):
    """2^22 rows, the most there may be: 131072 sequences of 32 tokens, one page each, heads of two dims; then one token for each."""
    B, n, D = 1 << 17, 32, 2
    g = torch.Generator(device="cuda").manual_seed(5)
    qkv = torch.empty((B * n, 3 * D), device="cuda").normal_(generator=g)
    k, v = gpu_lib.kv_cache(B, 32, 1, D)
    table = torch.randperm(B, device="cuda", generator=g).to(torch.int32)[:, None].contiguous()
    start = torch.arange(B + 1, device="cuda", dtype=torch.int32) * n
    lens = torch.full((B,), n, dtype=torch.int32, device="cuda")
    q = gpu_lib.rope_kv_append(qkv, None, k, v, table, lens, 1, q_start=start)
    assert torch.equal(q[:, 0], qkv[:, :D].to(torch.bfloat16))
    at = table[:, 0].long()
    keys, values = whole(k, 1, D, False)[at, 0], whole(v, 1, D, True)[at, 0]
    rounded = qkv.to(torch.bfloat16).double().reshape(B, n, 3, D)
    assert torch.equal(keys, rounded[:, :, 1]) and torch.equal(values, rounded[:, :, 2])
    y = gpu_lib.attention_prefill(q, k, v, table, lens, start, y_dtype=gpu_lib.F32)
    one = gpu_lib.attention_decode(q[n - 1::n].contiguous(), k, v, table, lens, y_dtype=gpu_lib.F32)
    qs = q.double().reshape(B, n, D)
    for b in range(0, B, 1 << 14):
        part = slice(b, b + (1 << 14))
        o, off = causal(qs[part], keys[part], values[part], D ** -0.5)
        assert bool(((y.double().reshape(B, n, D)[part] - o).abs() <= off).all())
        assert bool(((one.double()[part] - o[:, -1]).abs() <= off[:, -1]).all())


@pytest.mark.parametrize("D", [2, 8])
def test_positions_up_to_the_limit(gpu_lib, D):
    """A table of 2047 pages of 2^20 tokens, all but the last not there: the last 100 positions that a sequence can have."""
    P, per, kv_heads, heads, n = 1 << 20, 2047, 1, 2, 100
    end = per * P
    table = np.full((1, per), -1, dtype=np.int32)
    table[0, -1] = 0
    k, v = gpu_lib.kv_cache(1, P, kv_heads, D)
    k.fill_(float("nan")), v.fill_(float("nan"))
    rng = np.random.default_rng(64)
    x = bf16(rng.standard_normal((n, heads + 2 * kv_heads, D)))
    freq = np.array([0.5 ** i for i in range(D // 2)], dtype=np.float32)
    tab, lens = dev(table), dev([end])
    # the page's other tokens, up to the first of the 100, are there with keys and values of zero
    zeros = torch.zeros((P - n, (heads + 2 * kv_heads) * D), dtype=torch.bfloat16, device="cuda")
    gpu_lib.rope_kv_append(zeros, None, k, v, tab, dev([end - n]), heads, q_start=dev([0, P - n]))
    q = gpu_lib.rope_kv_append(dev16(x.reshape(n, -1)), dev(freq, np.float32), k, v, tab, lens, heads, q_start=dev([0, n]))
    angle = np.arange(end - n, end, dtype=np.float64)[:, None, None] * freq.astype(np.float64)
    a, b = x[:, : heads + 1, : D // 2], x[:, : heads + 1, D // 2:]
    turned = np.concatenate([a * np.cos(angle) - b * np.sin(angle), b * np.cos(angle) + a * np.sin(angle)], axis=-1)
    size = np.tile(np.abs(a) + np.abs(b), 2)
    off = size * 2.0 ** -20 + BF16_HALF_STEP * np.abs(turned) * 1.01
    qs = host(q)
    assert np.all(np.abs(qs - turned[:, :heads]) <= off[:, :heads])
    t = np.arange(P - n, P)
    j = t % 32
    key = host(k[0, 0, :, 0])[t // 32, 16 * ((j >> 2) & 1) + 4 * (j >> 3) + (j & 3), :D]
    assert np.all(np.abs(key - turned[:, heads]) <= off[:, heads])
    one = gpu_lib.attention_decode(q[-1:].contiguous(), k, v, tab, lens, y_dtype=gpu_lib.F32)
    y = gpu_lib.attention_prefill(q, k, v, tab, lens, dev([0, n]), y_dtype=gpu_lib.F32)
    values = x[:, -1]
    scale = D ** -0.5
    for r in (0, 37, n - 1):
        for h in range(heads):
            # P - n keys of zero have scores of zero and values of zero
            s = key[: r + 1] @ qs[r, h] * scale
            m = max(s.max(), 0.0)
            p, rest = np.exp(s - m), (P - n) * np.exp(-m)
            o, weight = p @ values[: r + 1] / (p.sum() + rest), p @ np.abs(values[: r + 1]) / (p.sum() + rest)
            # the sum of P weights: lanes, waves and workgroups have shares of it, of at most P terms
            by = 2 * (D + 8) * F32_HALF_STEP * scale * (np.abs(key) @ np.abs(qs[r, h])).max() + (2 * n + 64) * F32_HALF_STEP + BF16_HALF_STEP ** 2
            bound = weight * by * 1.01 + np.abs(o) * P * F32_HALF_STEP
            got = host(y)[r].reshape(heads, D)[h]
            assert np.all(np.abs(got - o) <= bound), (r, h)
            if r == n - 1:
                assert np.all(np.abs(host(one)[0].reshape(heads, D)[h] - o) <= bound), h
