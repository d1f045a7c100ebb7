"""What the cache's operators of a serving loop refuse, on the host and before anything is launched (the pointers here name no memory); and the host rule of
which tokens a sequence shares."""
import ctypes

import pytest
import torch

from paper_2402_17764_amd import binding as B
from test_attention_refusals_cpu import A, ALIGN, BAD, DTYPE, NULL, ODD, SHAPE, kv

WORKSPACE = 6
BIG = 1 << 40


def norm_append(c, qkv=A, dt=0, norm=1, qg=A, kg=A, eps=1e-6, freq=A, rotary=128, shift=A, T=3, heads=4, q=A):
    return B.load().bitnet_norm_rope_kv_append(qkv, dt, norm, qg, kg, eps, freq, rotary, 0, shift, c, T, heads, q, None)


def shared(c, q=A, start=A, length=A, prefixes=1, heads=4, scale=0.1, o=A, dt=0, ws=A, n=BIG):
    return B.load().bitnet_attention_decode_shared(q, c, start, length, prefixes, heads, scale, o, dt, ws, n, None)


def decode(c, q=A, heads=4, scale=0.1, o=A, dt=0, w=A, stride=256, ws=A, n=BIG):
    return B.load().bitnet_attention_decode_weights(q, c, heads, scale, o, dt, w, stride, ws, n, None)


def prefill(c, q=A, T=3, heads=4, scale=0.1, o=A, dt=0, w=A, stride=256, ws=A, n=BIG):
    return B.load().bitnet_attention_prefill_weights(q, c, T, heads, scale, o, dt, w, stride, ws, n, None)


def evict(c, w=A, stride=256, keep=100, recent=10, table=A, table_stride=2, w_out=0x2000, stride_out=128, lens=A, kept=A):
    return B.load().bitnet_kv_evict(c, w, stride, keep, recent, table, table_stride, w_out, stride_out, lens, kept, None)


ALL = (norm_append, shared, decode, prefill, evict)
ATTENTION = (shared, decode, prefill)


@pytest.mark.parametrize("change,status", BAD)
def test_caches_and_sequences(change, status):
    for call in ALL:
        if change != dict(kv_heads=3) or call is not evict:      # which has no query heads
            assert call(kv(**change)) == status


def test_no_cache_at_all():
    for call in ALL:
        assert call(None) == NULL


@pytest.mark.parametrize("heads", [0, -4, 3, 16386, 1 << 40])
def test_heads(heads):
    for call in ALL[:-1]:
        assert call(kv(), heads=heads) == SHAPE


def test_rows():
    for T in (0, -1, (1 << 22) + 1, 1 << 40):
        assert norm_append(kv(), T=T) == SHAPE and prefill(kv(), T=T) == SHAPE
    assert prefill(kv(), T=1 << 20, heads=256) == SHAPE
    assert norm_append(kv(q_start=None), T=4) == SHAPE
    assert prefill(kv(q_start=None)) == NULL


def test_norm_append_arguments():
    assert norm_append(kv(), qkv=None) == NULL and norm_append(kv(), q=None) == NULL and norm_append(kv(), freq=None) == NULL
    for rotary in (-2, 3, 130, 1 << 40):
        assert norm_append(kv(), rotary=rotary) == SHAPE
    for eps in (-1e-6, float("nan"), float("inf")):
        assert norm_append(kv(), eps=eps) == SHAPE
    assert norm_append(kv(), dt=2) == DTYPE and norm_append(kv(), dt=77) == DTYPE
    for bad in (dict(qkv=ODD), dict(qkv=0x1001, dt=1), dict(q=0x1001), dict(freq=ODD), dict(shift=ODD), dict(qg=ODD), dict(kg=ODD)):
        assert norm_append(kv(), **bad) == ALIGN


@pytest.mark.parametrize("call", ATTENTION)
def test_attention_arguments(call):
    assert call(kv(), q=None) == NULL and call(kv(), o=None) == NULL and call(kv(), ws=None) == NULL
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert call(kv(), scale=scale) == SHAPE
    assert call(kv(), dt=2) == DTYPE and call(kv(), dt=9) == DTYPE
    assert call(kv(), q=0x1001) == ALIGN and call(kv(), o=ODD) == ALIGN and call(kv(), o=0x1001, dt=1) == ALIGN and call(kv(), ws=0x1008) == ALIGN
    for n in (0, 16):
        assert call(kv(), n=n) == WORKSPACE


def test_shared_arguments():
    assert shared(kv(), start=None) == NULL and shared(kv(), length=None) == NULL
    assert shared(kv(), start=ODD) == ALIGN and shared(kv(), length=ODD) == ALIGN
    for prefixes in (0, -1, 1 << 22, 1 << 62):
        assert shared(kv(), prefixes=prefixes) == SHAPE


@pytest.mark.parametrize("call", (decode, prefill, evict))
def test_weights(call):
    assert call(kv(), w=None) == NULL
    for stride in (255, 0, -256, 1 << 62):
        assert call(kv(), stride=stride) == SHAPE
    assert call(kv(), w=ODD) == ALIGN


def test_evict_arguments():
    for name in ("table", "w_out", "lens", "kept"):
        assert evict(kv(), **{name: None}) == NULL and evict(kv(), **{name: ODD}) == ALIGN
    for keep in (0, -1, (1 << 31) - 64, 1 << 62):
        assert evict(kv(), keep=keep, recent=0) == SHAPE
    for recent in (-1, 101, 1 << 62):
        assert evict(kv(), recent=recent) == SHAPE
    assert evict(kv(), table_stride=1) == SHAPE and evict(kv(), table_stride=1 << 62) == SHAPE
    assert evict(kv(), stride_out=99) == SHAPE and evict(kv(), stride_out=1 << 62) == SHAPE
    assert evict(kv(), w_out=A, stride_out=300) == SHAPE              # in place with another stride


def test_sizes_of_workspaces():
    n = ctypes.c_size_t(0)
    f = B.load().bitnet_attention_shared_workspace
    assert f(kv(), 1, 4, 1, None) == NULL and f(None, 1, 4, 1, ctypes.byref(n)) == NULL
    for prefixes, heads in ((0, 4), (1 << 22, 4), (1, 3)):
        assert f(kv(), prefixes, heads, 1, ctypes.byref(n)) == SHAPE
    assert f(kv(), 2, 4, 2, ctypes.byref(n)) == DTYPE
    for dt in (0, 1):
        assert f(kv(), 2, 4, dt, ctypes.byref(n)) == 0 and n.value % 16 == 0 and 0 < n.value < 64 << 20
    f = B.load().bitnet_attention_weights_workspace
    assert f(kv(), 3, 4, 0, 1, None) == NULL and f(None, 3, 4, 0, 1, ctypes.byref(n)) == NULL and f(kv(), 0, 4, 1, 1, ctypes.byref(n)) == SHAPE
    assert f(kv(), 3, 4, 0, 2, ctypes.byref(n)) == DTYPE
    for p in (0, 1):
        for dt in (0, 1):
            assert f(kv(), 3, 4, p, dt, ctypes.byref(n)) == 0 and n.value % 16 == 0 and 0 < n.value < 64 << 20


X = torch.zeros(2, 64)


@pytest.mark.parametrize("call", [lambda t: B.norm_rope_kv_append(t, t, t, t, t, t, 4), lambda t: B.attention_decode_shared(t, t, t, t, t, t, t),
                                  lambda t: B.attention_decode_weights(t, t, t, t, t, t), lambda t: B.attention_prefill_weights(t, t, t, t, t, t, t),
                                  lambda t: B.kv_evict(t, t, t, t, t, 4, 1, t)])
@pytest.mark.parametrize("arg", [X, X.to(torch.int32), None, 3, "x"])
def test_only_gpu_tensors(call, arg):
    with pytest.raises(TypeError, match="must be a CUDA/HIP tensor"):
        call(arg)
