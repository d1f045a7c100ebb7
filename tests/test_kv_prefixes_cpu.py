"""Which tokens of the paged cache a sequence shares (csrc/kv_layout.hpp, compiled for the host): the documented ones, and whatever starts and lengths hold, no
sequence, row or token out of bounds."""
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
static KvView view(int max_blocks, int B) { return KvView{nullptr, nullptr, nullptr, nullptr, nullptr, max_blocks, 1, 1, max_blocks, max_blocks, 1, 64, B}; }
extern "C" int shared(const int32_t* start, const int32_t* len, int groups, int max_blocks, int B, int b, int tokens) {
    return shared_tokens(view(max_blocks, B), Prefixes{start, len, groups}, b, tokens);
}
extern "C" void rows(const int32_t* start, const int32_t* len, int groups, int max_blocks, int B, int i, int* out) {
    const SharedRows r(view(max_blocks, B), Prefixes{start, len, groups}, i);
    out[0] = r.first; out[1] = r.n; out[2] = r.len;
}
"""


@pytest.fixture(scope="module")
def rule(tmp_path_factory):
    d = tmp_path_factory.mktemp("kv_prefixes")
    src, lib = os.path.join(d, "shim.cpp"), os.path.join(d, "shim.so")
    with open(src, "w") as f:
        f.write(SHIM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-fsanitize=undefined", "-fsanitize-undefined-trap-on-error", "-fPIC", "-shared",
                           "-I", CSRC, src, "-o", lib])
    return ctypes.CDLL(lib)


def ints(a):
    a = np.ascontiguousarray(a, dtype=np.int32)
    return a, a.ctypes.data_as(ctypes.c_void_p)


def test_runs_that_do_not_fall(rule):
    rng = random.Random(5)
    for _ in range(400):
        B, groups, blocks = rng.randint(1, 30), rng.randint(1, 12), rng.randint(1, 40)
        starts = sorted(rng.randint(0, B) for _ in range(groups + 1))
        lens = [rng.randint(-50, 40 * 32 + 50) for _ in range(groups)]
        (s, sp), (n, np_) = ints(starts), ints(lens)
        for b in range(B):
            tokens = rng.randint(0, blocks * 32)
            i = next((i for i in range(groups) if starts[i] <= b < starts[i + 1]), None)
            want = 0 if i is None else min(tokens, max(0, min(lens[i], blocks * 32)))
            assert rule.shared(sp, np_, groups, blocks, B, b, tokens) == want
        out = (ctypes.c_int * 3)()
        for i in range(groups):
            rule.rows(sp, np_, groups, blocks, B, i, out)
            assert list(out) == [starts[i], starts[i + 1] - starts[i], max(0, min(lens[i], blocks * 32))]


def test_any_contents(rule):
    rng = random.Random(6)
    wild = [-2 ** 31, -1, 0, 1, 5, 2 ** 31 - 1]
    out = (ctypes.c_int * 3)()
    for _ in range(2000):
        B, groups, blocks = rng.randint(1, 12), rng.randint(1, 8), rng.randint(1, 9)
        (s, sp), (n, np_) = ints([rng.choice(wild + [rng.randint(-3, B + 3)]) for _ in range(groups + 1)]), ints([rng.choice(wild + [rng.randint(-9, 300)]) for _ in range(groups)])
        for b in range(B):
            tokens = rng.randint(0, blocks * 32)
            assert 0 <= rule.shared(sp, np_, groups, blocks, B, b, tokens) <= tokens
        for i in range(groups):
            rule.rows(sp, np_, groups, blocks, B, i, out)
            assert 0 <= out[0] and 0 <= out[1] and out[0] + out[1] <= B and 0 <= out[2] <= blocks * 32
