"""The exact search of token_topk (csrc/kth_key.hpp, which has no device code), without a GPU: what it finds, and that its counts
go through two buffers by turns."""
import ctypes
import functools
import os
import random
import subprocess
import tempfile

import pytest

from paper_2507_19766_amd import build

_SOURCE = """
#include "kth_key.hpp"
extern "C" unsigned long search(unsigned K, unsigned n, const unsigned long* keys, long count, int* turns, int* calls)
{
    *calls = 0;
    return ulorl_detail::kth_key(K, n, [&](uint64_t c, int turn) {
        turns[(*calls)++] = turn;
        uint32_t reach = 0;
        for (long i = 0; i < count; ++i) reach += keys[i] >= c ? 1u : 0u;
        return reach;
    });
}
"""


@functools.lru_cache(None)
def _library():
    with tempfile.TemporaryDirectory() as tmp:
        src, lib = os.path.join(tmp, "search.cpp"), os.path.join(tmp, "search.so")
        with open(src, "w") as f:
            f.write(_SOURCE)
        subprocess.check_call(["g++", "-O1", "-std=c++17", "-Wall", "-fPIC", "-shared", "-I" + build.CSRC, src, "-o", lib])
        found = ctypes.CDLL(lib)
    found.search.restype = ctypes.c_ulong
    return found


def search(K, n, keys):
    turns, calls = (ctypes.c_int * 64)(), ctypes.c_int()
    t = _library().search(K, n, (ctypes.c_ulong * len(keys))(*keys), len(keys), turns, ctypes.byref(calls))
    return t, list(turns[:calls.value])


def key(order, i):
    return order << 32 | (0xffffffff - i)


@pytest.mark.parametrize("id_bits", range(1, 32))
def test_every_count_takes_the_other_buffer_than_the_one_before(id_bits):
    """Also where the search goes on below the logits' order, past the bits that no id has: equal logits, and fewer keys than K."""
    for n in {1 << (id_bits - 1), (1 << id_bits) - 1}:
        ids = sorted(random.Random(id_bits).sample(range(n), min(n, 40)))
        for K in (1, 2, 5, len(ids), len(ids) + 1):
            for keys in ([key(0xbfc00000, i) for i in ids], [key(0x80000000 + i % 3, i) for i in ids], [0] * 10):
                _, turns = search(K, n, keys)
                assert len(turns) and all((a ^ b) & 1 for a, b in zip(turns, turns[1:])), (n, K, turns)


@pytest.mark.parametrize("n", [1, 2, 100, 125, 1000, 4096, 32003, 65535, 128256, 151936, 2 ** 31 - 1])
def test_k_keys_reach_what_is_found(n):
    r = random.Random(n)
    for orders in ([7], [0x80000000, 0x80000001], range(1, 1 << 32, 12345677), [0, 0, 0, 0xc0000000]):
        ids = r.sample(range(n), min(n, 300))
        keys = [key(o, i) if o else 0 for o, i in ((r.choice(orders), i) for i in ids)]
        live = sorted((k for k in keys if k), reverse=True)
        for K in (1, 2, 33, 128):
            t, _ = search(K, n, keys)
            assert [k for k in live if k >= t] == live[:K]
