"""Every form of the kernels over shared prefixes and of those that add up weights that a head's size, the rows of a group and a call's length choose.  The
definition and the bounds are attention_ref's and cache_ref's; long runs are reckoned in 64 bits on the device."""
import numpy as np
import pytest

from attention_ref import F32_HALF_STEP
from test_gpu_attention import Batch, check_attention, dev, dev16, host
from test_gpu_cache_ops import run_norm_append, run_shared, run_weights

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# one size at least for each built form: chunks of 32 dims that are whole (32 ... 256), and filled in part with one tile of 16 dims in the last
# chunk or two; up to 62 dims a stage is two blocks of the cache
FORMS = [2, 16, 30, 32, 40, 48, 56, 62, 64, 80, 90, 96, 98, 112, 120, 126, 128, 130, 160, 190, 192, 194, 250, 256]


@pytest.mark.parametrize("D", FORMS)
@pytest.mark.parametrize("f32", [False, True])
def test_shared_groups_of_few_and_of_many_rows(gpu_lib, D, f32):
    """6, 192 and 320 rows a key-value head: one launch, two, and tiles of 128 rows where a bf16 result of up to 128 dims takes them."""
    run_shared(gpu_lib, [700, 641, 600, 900, 5, 1300], [4, 2], [640, 3], 2, 2, D, 96, f32, seed=31)
    run_shared(gpu_lib, [700 + 3 * (b % 7) for b in range(24)], [24], [650], 16, 2, D, 96, f32, seed=32, rows=5)
    run_shared(gpu_lib, [700 + 90 * (b % 7) - 600 * (b % 13 == 12) for b in range(40)], [40], [650], 16, 2, D, 32, f32, seed=33, rows=6)


@pytest.mark.parametrize("D", FORMS)
@pytest.mark.parametrize("f32", [False, True])
def test_decode_weights(gpu_lib, D, f32):
    run_weights(gpu_lib, [(1499, 1), (30, 1), (777, 1)], 6, 2, D, 32, f32, True, seed=34)


@pytest.mark.parametrize("D", FORMS)
@pytest.mark.parametrize("f32", [False, True])
def test_prefill_weights(gpu_lib, D, f32):
    """Rows and keys that workgroups share; tiles of 64 rows."""
    run_weights(gpu_lib, [(1500, 5), (0, 3), (255, 1)], 6, 2, D, 32, f32, False, seed=35, first=1, behind=2)
    run_weights(gpu_lib, [(0, 150), (300, 70)], 4, 2, D, 96, f32, False, seed=36, rows=20)


def long_run(gpu_lib, old, n, heads, kv_heads, D, P, f32, seed):
    batch = Batch([old + n], P, kv_heads, D, seed)
    q = batch.queries(n, heads, D)
    acc = torch.rand((1, kv_heads, batch.per * P), device="cuda")
    was, qd, scale = acc.clone(), dev16(q), D ** -0.5
    y = gpu_lib.attention_prefill_weights(qd, batch.k, batch.v, dev(batch.table), dev([old + n]), dev([0, n]), acc, y_dtype=gpu_lib.F32 if f32 else gpu_lib.BF16)
    at = sorted({0, n - 1} | set(int(i) for i in batch.rng.integers(0, n, 8)))
    check_attention(host(y)[at], q[at], batch, [(0, old + i) for i in at], scale, f32)
    keys = torch.from_numpy(batch.cache.get(batch.table[0], old + n)[0]).cuda()
    g = heads // kv_heads
    for h in sorted({0, kv_heads - 1}):
        rows = qd[:, h * g: h * g + g].double().reshape(n * g, D)
        hidden = torch.arange(old + n, device="cuda")[None] > (old + torch.arange(n, device="cuda")).repeat_interleave(g)[:, None]
        p = torch.softmax((rows @ keys[:, h].t() * scale).masked_fill_(hidden, -float("inf")), dim=1)
        # cache_ref's bound of a row: scores, the sum that divides it, the sum over the rows
        by = 2 * (D + 8) * F32_HALF_STEP * scale * (rows.abs() @ keys[:, h].abs().t()).masked_fill_(hidden, 0).amax(dim=1) + (old + n + 64) * F32_HALF_STEP
        want, off = p.sum(dim=0), (p * by[:, None]).sum(dim=0) * 1.01
        want[:old] += was[0, h, :old].double()
        off += (n * g + 2) * F32_HALF_STEP * want
        assert ((acc[0, h, : old + n].double() - want).abs() <= off).all(), h
    assert torch.equal(acc[0, :, old + n:], was[0, :, old + n:])


@pytest.mark.parametrize("D", FORMS)
@pytest.mark.parametrize("f32", [False, True])
def test_prefill_weights_of_long_runs(gpu_lib, D, f32):
    """A chunk behind others in tiles of 128 rows; a prompt whose tiles of keys go to many workgroups."""
    long_run(gpu_lib, 3200, 1030, 64, 8, D, 96, f32, 37)
    long_run(gpu_lib, 0, 700, 8, 1, D, 32, f32, 38)


@pytest.mark.parametrize("rotary,D", [(d, d) for d in FORMS] + [(16, 64), (48, 128), (2, 130), (34, 256), (256, 256), (226, 230)])
@pytest.mark.parametrize("f32", [False, True])
def test_norm_append(gpu_lib, rotary, D, f32):
    """Slots of a head in 8, 16 and 32 lanes, each way of turning, workgroups of one head and of several."""
    for pairs in (False, True):
        run_norm_append(gpu_lib, [(3, 40), (70, 1), (0, 33)], 4, 2, D, 32, f32, pairs, rotary=rotary, seed=39, shift=[5, 0, 100])
        run_norm_append(gpu_lib, [(31, 300)] * 6, 10, 5, D, 64, f32, pairs, rotary=rotary, seed=39)
