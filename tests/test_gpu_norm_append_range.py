"""The norm of norm_rope_kv_append at the ends of its arithmetic: sums of squares in 64 bits, whichever kernel takes a row."""
import numpy as np
import pytest

from attention_ref import F32_HALF_STEP
from test_gpu_attention import dev, host

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def nearest_bf16(x):
    """fp64 -> the nearest bf16 in one step (eight bits, ties to even), for numbers that are normal ones there."""
    m, e = np.frexp(x)
    return np.ldexp(np.rint(m * 256.0), e - 8)


def append(gpu_lib, x, D, one, q_gain=None, eps=0.0, freq=None, k_gain=None):
    """x [n, 3, D] fp32: a query, a key and a value head of n sequences' first tokens -> (queries [n, D], keys [n, D]) on the host."""
    n = len(x)
    k, v = gpu_lib.kv_cache(n, 32, 1, D)
    k.fill_(1.0), v.fill_(1.0)
    as_dev = lambda a: None if a is None else dev(a, np.float32)  # noqa: E731
    q = gpu_lib.norm_rope_kv_append(dev(x.reshape(n, -1), np.float32), as_dev(freq), k, v, torch.arange(n, device="cuda", dtype=torch.int32).view(n, 1), dev(np.ones(n)), 1,
                                    as_dev(q_gain), as_dev(k_gain), eps, q_start=None if one else dev(np.arange(n + 1)))
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
