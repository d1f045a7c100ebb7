"""What the attention half of the library refuses, on the host and before anything is launched (the pointers here name no memory)."""
import ctypes

import pytest
import torch

from paper_2402_17764_amd import binding as B

A, ODD = 0x1000, 0x1002
NULL, SHAPE, DTYPE, ALIGN = 1, 2, 3, 5


def kv(**change):
    f = dict(k=A, v=A, pages=10, page_tokens=64, kv_heads=2, head_dim=128, sequences=3, page_table=A, table_stride=4, max_pages=4, kv_len=A, q_start=A)
    f.update(change)
    return ctypes.byref(B.KvStruct(**f))


BAD = [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(page_table=None), NULL), (dict(kv_len=None), NULL),
    (dict(k=ODD), ALIGN), (dict(v=0x1008), ALIGN), (dict(page_table=ODD), ALIGN), (dict(kv_len=ODD), ALIGN), (dict(q_start=ODD), ALIGN),
    (dict(pages=0), SHAPE), (dict(pages=-1), SHAPE), (dict(pages=1 << 30), SHAPE), (dict(pages=1 << 62), SHAPE),
    (dict(page_tokens=0), SHAPE), (dict(page_tokens=16), SHAPE), (dict(page_tokens=65), SHAPE), (dict(page_tokens=1 << 40), SHAPE),
    (dict(kv_heads=0), SHAPE), (dict(kv_heads=3), SHAPE), (dict(kv_heads=1 << 33), SHAPE),
    (dict(head_dim=0), SHAPE), (dict(head_dim=63), SHAPE), (dict(head_dim=258), SHAPE), (dict(head_dim=-2), SHAPE),
    (dict(sequences=0), SHAPE), (dict(sequences=1 << 22), SHAPE), (dict(sequences=1 << 62), SHAPE),
    (dict(max_pages=0), SHAPE), (dict(table_stride=3), SHAPE), (dict(table_stride=1 << 62), SHAPE), (dict(max_pages=1 << 26, table_stride=1 << 26), SHAPE),
    (dict(max_pages=1 << 62, table_stride=1 << 62), SHAPE), (dict(sequences=1 << 19, max_pages=1 << 20, table_stride=1 << 20), SHAPE),
]


def append(c, qkv=A, dt=0, freq=A, rotary=128, T=3, heads=4, q=A):
    return B.load().bitnet_rope_kv_append(qkv, dt, freq, rotary, 0, c, T, heads, q, None)


def decode(c, q=A, heads=4, scale=0.1, o=A, dt=0, ws=None, n=0):
    return B.load().bitnet_attention_decode(q, c, heads, scale, o, dt, ws, n, None)


def prefill(c, q=A, T=3, heads=4, scale=0.1, o=A, dt=0, ws=None, n=0):
    return B.load().bitnet_attention_prefill(q, c, T, heads, scale, o, dt, ws, n, None)


@pytest.mark.parametrize("change,status", BAD)
def test_caches_and_sequences(change, status):
    for call in (append, decode, prefill):
        assert call(kv(**change)) == status


def test_no_cache_at_all():
    for call in (append, decode, prefill):
        assert call(None) == NULL


@pytest.mark.parametrize("heads", [0, -4, 3, 16386, 1 << 40])
def test_heads(heads):
    for call in (append, decode, prefill):
        assert call(kv(), heads=heads) == SHAPE


def test_rows():
    for T in (0, -1, (1 << 22) + 1, 1 << 40):
        assert append(kv(), T=T) == SHAPE and prefill(kv(), T=T) == SHAPE
    assert prefill(kv(), T=1 << 20, heads=256) == SHAPE              # rows times heads
    assert append(kv(q_start=None), T=4) == SHAPE                   # one row for each sequence
    assert prefill(kv(q_start=None)) == NULL


def test_append_arguments():
    assert append(kv(), qkv=None) == NULL and append(kv(), q=None) == NULL and append(kv(), freq=None) == NULL
    for rotary in (-2, 3, 130, 1 << 40):
        assert append(kv(), rotary=rotary) == SHAPE
    assert append(kv(), dt=2) == DTYPE and append(kv(), dt=77) == DTYPE
    assert append(kv(), qkv=ODD) == ALIGN and append(kv(), qkv=0x1001, dt=1) == ALIGN and append(kv(), q=0x1001) == ALIGN and append(kv(), freq=ODD) == ALIGN


@pytest.mark.parametrize("call", [decode, prefill])
def test_attention_arguments(call):
    assert call(kv(), q=None) == NULL and call(kv(), o=None) == NULL
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert call(kv(), scale=scale) == SHAPE
    assert call(kv(), dt=2) == DTYPE and call(kv(), dt=9) == DTYPE
    assert call(kv(), q=0x1001) == ALIGN and call(kv(), o=ODD) == ALIGN and call(kv(), o=0x1001, dt=1) == ALIGN and call(kv(), ws=0x1008, n=1 << 20) == ALIGN


def test_sizes_of_caches_and_workspaces():
    n = ctypes.c_size_t(0)
    f = B.load().bitnet_kv_cache_bytes
    assert f(10, 64, 2, 100, ctypes.byref(n)) == 0 and n.value == 10 * 64 * 2 * 104 * 2
    assert f(1, 32, 1, 2, ctypes.byref(n)) == 0 and n.value == 32 * 8 * 2
    assert f(10, 64, 2, 100, None) == NULL
    for bad in ((0, 64, 2, 64), (1, 48, 2, 64), (1, 64, 0, 64), (1, 64, 1, 257), (1 << 31, 32, 1, 64), (1 << 62, 32, 1, 64)):
        assert f(*bad, ctypes.byref(n)) == SHAPE
    w = B.load().bitnet_attention_workspace
    assert w(kv(), 3, 4, 0, None) == NULL and w(None, 3, 4, 0, ctypes.byref(n)) == NULL and w(kv(), 0, 4, 1, ctypes.byref(n)) == SHAPE
    for p in (0, 1):
        assert w(kv(), 3, 4, p, ctypes.byref(n)) == 0 and n.value % 16 == 0 and n.value < 64 << 20


X = torch.zeros(2, 64)


@pytest.mark.parametrize("call", [lambda t: B.rope_kv_append(t, t, t, t, t, t, 4), lambda t: B.attention_decode(t, t, t, t, t),
                                  lambda t: B.attention_prefill(t, t, t, t, t, t)])
@pytest.mark.parametrize("arg", [X, X.to(torch.int32), None, 3, "x"])
def test_only_gpu_tensors(call, arg):
    with pytest.raises(TypeError, match="must be a CUDA/HIP tensor"):
        call(arg)
