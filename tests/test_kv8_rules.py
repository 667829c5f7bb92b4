"""How attention over the 8-bit cache is divided (csrc/kv8_rules.hpp), compiled
for the host: every key of a segment falls into one chunk, and partial results
fit the workspace whatever part of the tokens counts."""
import ctypes
import functools
import os
import subprocess
import tempfile

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include <string.h>
#include "kv8_rules.hpp"
extern "C" void plan(int heads, int nseg, const int64_t* rows, const int* klen, int* chunk, int* chunks, int* item,
                     int* row, int64_t* part) {
  const sphinx::Kv8Plan p = sphinx::plan_kv8(heads, nseg, rows, klen);
  *chunk = p.chunk;
  memcpy(chunks, p.chunks, 4 * nseg);
  memcpy(item, p.item, 4 * (nseg + 1));
  memcpy(row, p.row, 4 * (nseg + 1));
  memcpy(part, p.part, 8 * (nseg + 1));
}
extern "C" int64_t most(int heads, int nseg, const int64_t* rows, const int* klen) {
  return sphinx::kv8_most_parts(heads, nseg, rows, klen);
}
extern "C" int tile(int64_t rows) { return sphinx::kv8_tiles(rows); }
"""


@functools.lru_cache(None)
def lib():
    with tempfile.TemporaryDirectory() as d:
        src, out = os.path.join(d, "rules.cpp"), os.path.join(d, "rules.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC",
                        "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2511_18672_amd", "csrc"),
                        src, "-o", out], check=True)
        L = ctypes.CDLL(out)
        L.most.restype = ctypes.c_int64
        return L


def ptr(a):
    return a.ctypes.data_as(ctypes.c_void_p)


def plan(heads, rows, klen):
    n = len(rows)
    rows, klen = np.ascontiguousarray(rows, np.int64), np.ascontiguousarray(klen, np.int32)
    chunk = np.zeros(1, np.int32)
    out = [np.zeros(n, np.int32), np.zeros(n + 1, np.int32), np.zeros(n + 1, np.int32), np.zeros(n + 1, np.int64)]
    lib().plan(heads, n, ptr(rows), ptr(klen), ptr(chunk), *(ptr(a) for a in out))
    return (int(chunk[0]), *out)


def most(heads, rows, klen):
    return lib().most(heads, len(rows), ptr(np.ascontiguousarray(rows, np.int64)),
                      ptr(np.ascontiguousarray(klen, np.int32)))


@pytest.mark.parametrize("seed", range(40))
def test_plan_covers_every_key_once_and_fits_its_workspace(seed):
    rng = np.random.default_rng(seed)
    n = int(rng.integers(1, 65))
    heads = int(rng.choice([1, 2, 5, 16, 64]))
    rows = np.exp(rng.uniform(0, np.log(rng.choice([4, 200, 30000])), n)).astype(np.int64)
    cap = np.exp(rng.uniform(0, np.log(rng.choice([100, 30000, 4000000])), n)).astype(np.int64)
    bound = most(heads, rows, cap)
    for klen in (cap, (cap * rng.random(n)).astype(np.int64), cap * (rng.random(n) < 0.2)):
        chunk, chunks, item, row, part = plan(heads, rows, klen)
        blocks = (klen + 63) // 64
        assert chunk >= 4 and (chunks >= 1).all()
        # the last chunk of a segment holds a block, and the chunks together hold all of them
        assert (chunks * chunk >= blocks).all() and (((chunks - 1) * chunk < blocks) | (chunks == 1)).all()
        split = chunks > 1
        assert np.array_equal(np.diff(row), np.where(split, rows, 0)) and row[0] == 0
        assert np.array_equal(np.diff(part), np.where(split, rows * heads * chunks, 0)) and part[0] == 0
        tiles = np.diff(item) // chunks
        assert np.array_equal(np.diff(item), tiles * chunks)
        assert part[-1] <= bound
        # a call is not cut finer than its purpose asks
        assert (tiles * chunks * heads)[split].sum() <= 2048


def test_largest_calls_stay_in_range():
    rows = [(1 << 31) - 1]
    chunk, chunks, item, row, part = plan(1, rows, [(1 << 31) - 1])
    assert chunks[0] == 1 and item[1] == lib().tile(ctypes.c_int64(rows[0])) and part[1] == 0
    chunk, chunks, item, row, part = plan(1, [1], [(1 << 31) - 1])
    assert chunks[0] * chunk >= 1 << 25 and part[1] == chunks[0] <= most(1, [1], [(1 << 31) - 1])
