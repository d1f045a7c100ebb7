"""The norm of norm_rope_kv_append at the ends of its arithmetic: sums of squares in 64 bits, whichever kernel takes a row."""
import numpy as np
import pytest

from attention_ref import F32_HALF_STEP, bf16
from test_gpu_attention import dev, host

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def nearest_bf16(x):
    """fp64 -> the nearest bf16 in one step (eight bits, ties to even), for numbers that are normal ones there."""
    m, e = np.frexp(x)
    return np.ldexp(np.rint(m * 256.0), e - 8)


def append(gpu_lib, x, D, one, q_gain=None, eps=0.0, freq=None, k_gain=None, pairs=False, f32=True):
    """x [n, 3, D]: a query, a key and a value head of n sequences' first tokens -> (queries [n, D], keys [n, D]) on the host."""
    n = len(x)
    k, v = gpu_lib.kv_cache(n, 32, 1, D)
    k.fill_(1.0), v.fill_(1.0)
    as_dev = lambda a: None if a is None else dev(a, np.float32)  # noqa: E731
    qkv = dev(x.reshape(n, -1), np.float32).to(torch.float32 if f32 else torch.bfloat16)
    q = gpu_lib.norm_rope_kv_append(qkv, as_dev(freq), k, v, torch.arange(n, device="cuda", dtype=torch.int32).view(n, 1), dev(np.ones(n)), 1,
                                    as_dev(q_gain), as_dev(k_gain), eps, q_start=None if one else dev(np.arange(n + 1)), pairs=pairs)
    return host(q)[:, 0], host(k)[:, 0, 0, :, 0].reshape(n, -1)[:, :D]


@pytest.mark.parametrize("one", [False, True])
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("turned", [False, True])
def test_sums_of_squares_are_64_bits(gpu_lib, one, D, turned):
    """A one and small elements whose squares are just below its half step in 32 bits, where a sum of eight would lose seven of them: 3.5 half steps of the
    factor.  In 64 bits the factor has its rounding to fp32 and the two products one each, 3 half steps; a turn by position 0 adds none.  So the result
    is the rounding of some number that near the defined one."""
    rng = np.random.default_rng([17, D])
    n = 8192
    x = rng.uniform(0.90, 0.999, (n, 3, D)) * 2.0 ** -12 * rng.choice([-1.0, 1.0], (n, 3, D))
    x[..., 0] = 1.0
    x = x.astype(np.float32)
    gains = [rng.uniform(0.5, 2.0, D).astype(np.float32) for _ in range(2)]
    freq = np.ones(D // 2) if turned else None
    for got, i, gain in zip(append(gpu_lib, x, D, one, gains[0], 0.0, freq, gains[1]), (0, 1), gains):
        y = x[:, i].astype(np.float64)
        y = np.abs(y / np.sqrt((y * y).mean(axis=1, keepdims=True)) * gain.astype(np.float64))
        assert np.all(np.abs(got) >= nearest_bf16(y * (1 - 3.01 * F32_HALF_STEP))) and np.all(np.abs(got) <= nearest_bf16(y * (1 + 3.01 * F32_HALF_STEP)))


@pytest.mark.parametrize("one", [False, True])
@pytest.mark.parametrize("D", [8, 64, 100, 128, 256])
@pytest.mark.parametrize("turned", [None, "halves", "pairs"])
@pytest.mark.parametrize("f32", [False, True])
def test_heads_with_infinities(gpu_lib, one, D, turned, f32):
    """x / inf: zeros in the finite dims, no number in the others, nor in what they are turned with; a head that is no number somewhere is none anywhere.  The heads
    beside them are what they are without."""
    rng = np.random.default_rng(D)
    x = bf16(rng.standard_normal((5, 3, D)))
    plain = append(gpu_lib, x, D, one, eps=1e-6, freq=None if turned is None else np.ones(D // 2), pairs=turned == "pairs", f32=f32)
    marks = {(0, 0): {1: np.inf}, (0, 1): {D - 1: -np.inf}, (1, 0): {0: np.inf, D // 2: -np.inf}, (2, 1): {3: np.nan}, (3, 0): {2: np.inf, 5: np.nan}}
    for (b, i), at in marks.items():
        for d, value in at.items():
            x[b, i, d] = value
    got = append(gpu_lib, x, D, one, eps=1e-6, freq=None if turned is None else np.ones(D // 2), pairs=turned == "pairs", f32=f32)
    for b in range(5):
        for i in range(2):
            at = marks.get((b, i))
            if at is None:
                assert np.array_equal(got[i][b], plain[i][b])
                continue
            if any(np.isnan(value) for value in at.values()):
                assert np.isnan(got[i][b]).all()
                continue
            none = set(at) if turned is None else set(at) | {d ^ 1 if turned == "pairs" else (d + D // 2) % D for d in at}
            assert np.isnan(got[i][b][sorted(none)]).all() and (np.delete(got[i][b], sorted(none)) == 0).all()


@pytest.mark.parametrize("one", [False, True])
@pytest.mark.parametrize("size", [3e38, 1e25, 1e-19, 1e-30, 1e-37, 1e-39, 1e-41, 3e-44])
@pytest.mark.parametrize("turned", [None, "halves", "pairs"])
@pytest.mark.parametrize("f32", [False, True])
def test_heads_near_both_ends_of_the_range(gpu_lib, one, size, turned, f32):
    """Without eps a head of any size comes out as one of size one: the factor is rounded once, to fp32, and the two products are (a power of two in front of them
    changes nothing): 3 half steps, at position 0."""
    rng = np.random.default_rng(3)
    n, D = 1000, 128 if turned != "halves" else 100
    x = (rng.uniform(0.3, 1.0, (n, 3, D)) * rng.choice([-1.0, 1.0], (n, 3, D)) * size).astype(np.float32).astype(np.float64)
    if not f32:
        x = bf16(x)
    gains = [rng.uniform(0.5, 2.0, D).astype(np.float32) for _ in range(2)]
    got = append(gpu_lib, x, D, one, gains[0], 0.0, None if turned is None else np.ones(D // 2), gains[1], turned == "pairs", f32)
    for i, gain in enumerate(gains):
        y, some = x[:, i], x[:, i].any(axis=1)
        y = np.abs(y[some] / np.sqrt((y[some] * y[some]).mean(axis=1, keepdims=True)) * gain.astype(np.float64))
        assert some.any() or not f32
        assert np.all(np.abs(got[i][some]) >= nearest_bf16(y * (1 - 3.01 * F32_HALF_STEP))) and np.all(np.abs(got[i][some]) <= nearest_bf16(y * (1 + 3.01 * F32_HALF_STEP)))
        assert (got[i][~some] == 0).all()


@pytest.mark.parametrize("D", [8, 64, 100, 128, 256])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("f32", [False, True])
def test_a_row_of_a_prompt_is_the_token(gpu_lib, D, pairs, f32):
    """The same bits from both kernels: sums of squares in 64 bits differ by their order in 2^-50 of them, which reaches the factor's rounding to 24 bits
    in one of 2^26 heads."""
    rng = np.random.default_rng(D)
    n, heads, kv_heads = 1500, 4, 2
    x = rng.standard_normal((n, (heads + 2 * kv_heads) * D)) * np.exp(rng.standard_normal((n, 1)))
    qkv = dev(x, np.float32).to(torch.float32 if f32 else torch.bfloat16)
    freq, gains = dev(10000.0 ** (-np.arange(0, D, 2) / D), np.float32), [dev(rng.uniform(0.5, 2.0, D), np.float32) for _ in range(2)]
    table, lens = torch.arange(n, device="cuda", dtype=torch.int32).view(n, 1), dev(rng.integers(1, 33, n))
    got = []
    for start in (None, dev(np.arange(n + 1))):
        k, v = gpu_lib.kv_cache(n, 32, kv_heads, D)
        k.zero_(), v.zero_()
        got.append((gpu_lib.norm_rope_kv_append(qkv, freq, k, v, table, lens, heads, *gains, q_start=start, pairs=pairs), k, v))
    assert all(torch.equal(a, b) for a, b in zip(*got))
