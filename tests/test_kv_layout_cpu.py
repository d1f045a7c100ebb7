"""The index rules of the paged cache and of the tiles over ragged runs of rows (csrc/kv_layout.hpp, compiled for the host): the places
are those that bitnet.h documents, every element has one, and no page table, length or row start, whatever it holds, leads out of bounds."""
import ctypes
import os
import random
import subprocess

import numpy as np
import pytest

from paper_2402_17764_amd.build import CSRC

SHIM = """
#include "kv_layout.hpp"
using namespace bitnet;
extern "C" int key_at(int t, int d) { return kv_key_at(t, d); }
extern "C" int value_at(int t, int d, int Dp) { return kv_value_at(t, d, Dp); }
static KvView view(const int32_t* table, const int32_t* len, const int32_t* start, int pages, int page_blocks, int max_blocks, int heads, int B) {
    return KvView{nullptr, nullptr, table, len, start, max_blocks / page_blocks, pages, page_blocks, max_blocks / page_blocks, max_blocks, heads, 64, B};
}
extern "C" int block(const int32_t* row, int pages, int page_blocks, int max_blocks, int heads, int blk, int h) {
    return view(row, nullptr, nullptr, pages, page_blocks, max_blocks, heads, 1).block(row, blk, h);
}
extern "C" int length(int max_blocks, int len) { return view(nullptr, nullptr, nullptr, 1, 1, max_blocks, 1, 1).length(len); }
extern "C" void rows(const int32_t* len, const int32_t* start, int max_blocks, int B, int b, int T, int* out) {
    const NewTokens n(view(nullptr, len, start, 1, 1, max_blocks, 1, B), b, T);
    out[0] = n.first; out[1] = n.n; out[2] = n.pos0;
}
extern "C" int seq_of(const int32_t* start, int B, int64_t x, int each, int size, int extra) { return sequence_of_tile(start, B, x, each, size, extra); }
extern "C" int64_t tile0(int32_t start, int b, int each, int size, int extra) { return first_tile(start, b, each, size, extra); }
extern "C" int64_t tiles(int64_t T, int64_t B, int each, int size, int extra) { return tiles_at_most(T, B, each, size, extra); }
"""


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("kv_layout")
    src, lib = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fsanitize-undefined-trap-on-error", "-fPIC", "-shared",
                           "-I", CSRC, src, "-o", lib])
    so = ctypes.CDLL(lib)
    so.seq_of.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int64] + [ctypes.c_int] * 3
    so.tile0.restype = so.tiles.restype = ctypes.c_int64
    so.tiles.argtypes = [ctypes.c_int64, ctypes.c_int64] + [ctypes.c_int] * 3
    return so


def ints(a):
    a = np.ascontiguousarray(a, dtype=np.int32)
    return a, a.ctypes.data_as(ctypes.c_void_p)


@pytest.mark.parametrize("D", [2, 8, 64, 100, 128, 250, 256])
def test_places_are_the_documented_ones_and_each_is_taken_once(rule, D):
    Dp = (D + 7) // 8 * 8
    keys = [[rule.key_at(t, d) for d in range(Dp)] for t in range(32)]
    values = [[rule.value_at(t, d, Dp) for d in range(Dp)] for t in range(32)]
    assert sorted(sum(keys, [])) == list(range(32 * Dp)) == sorted(sum(values, []))
    for t in range(32):
        for d in range(Dp):
            assert keys[t][d] == (d // 8 * 32 + 16 * ((t >> 2) & 1) + 4 * (t >> 3) + (t & 3)) * 8 + d % 8
            assert values[t][d] == (t // 8 * Dp + d) * 8 + t % 8


def test_block_numbers_stay_in_the_cache(rule):
    rng = random.Random(5)
    big = (2 ** 31 - 1) // (8 * 4)
    for pages, page_blocks, heads in [(1, 1, 1), (7, 3, 5), (big, 4, 8)]:
        row, p = ints([rng.choice([0, pages - 1, rng.randrange(pages), -1, -2 ** 31, pages, 2 ** 31 - 1]) for _ in range(50)])
        for blk in range(50 * page_blocks):
            for h in (0, heads - 1):
                got = rule.block(p, pages, page_blocks, 50 * page_blocks, heads, blk, h)
                page = int(row[blk // page_blocks])
                assert got == ((page * heads + h) * page_blocks + blk % page_blocks if 0 <= page < pages else -1)
                assert got < pages * heads * page_blocks


def test_lengths_are_held_to_the_table(rule):
    for most in (1, 7, (2 ** 31 - 65) // 32):
        for n in (-2 ** 31, -1, 0, 1, 32 * most - 1, 32 * most, 32 * most + 1, 2 ** 31 - 1):
            assert rule.length(most, n) == min(max(n, 0), 32 * most) or n > 2 ** 31 - 1


@pytest.mark.parametrize("each,size,extra", [(1, 32, 2), (1, 64, 1), (8, 128, 1), (7, 128, 1), (12, 64, 1), (64, 256, 1)])
def test_every_tile_of_a_ragged_batch_is_dealt_out_once(rule, each, size, extra):
    rng = random.Random(each * size)
    for _ in range(200):
        B = rng.choice([1, 2, 3, 17, 100])
        n = [rng.choice([0, 0, 1, 2, 31, 32, 33, rng.randrange(400)]) for _ in range(B)]
        first = rng.choice([0, 0, 5])
        start, p = ints(np.cumsum([first] + n))
        T = int(start[-1]) + rng.choice([0, 9])
        total = rule.tiles(T, B, each, size, extra)
        for b in range(B):
            need = -(-n[b] * each // size) if extra == 1 else (0 if n[b] == 0 else (n[b] - 2) // 32 + 2 if n[b] > 1 else 1)
            x0 = rule.tile0(int(start[b]), b, each, size, extra)
            for x in range(x0, x0 + need):
                assert 0 <= x < total and rule.seq_of(p, B, x, each, size, extra) == b


def test_any_row_starts_stay_in_the_rows(rule):
    rng = random.Random(9)
    out = (ctypes.c_int * 3)()
    for _ in range(300):
        B, T, most = rng.choice([1, 4, 30]), rng.choice([1, 50, 2 ** 22]), rng.choice([1, 9, 2 ** 20])
        pick = lambda: rng.choice([0, 1, T, T + 1, -1, -2 ** 31, 2 ** 31 - 1, rng.randrange(T + 1)])  # noqa: E731
        start, p = ints([pick() for _ in range(B + 1)])
        lens, q = ints([rng.choice([0, 1, -5, 2 ** 31 - 1, rng.randrange(40 * most)]) for _ in range(B)])
        for b in range(B):
            rule.rows(q, p, most, B, b, T, out)
            first, n, pos0 = out
            assert 0 <= first <= T and 0 <= n <= T - first and -T <= pos0 and pos0 + n <= 32 * most
        for x in (0, 1, 7, 2 ** 40):
            for each, size, extra in ((1, 32, 2), (8, 128, 1)):
                assert 0 <= rule.seq_of(p, B, x, each, size, extra) < B
