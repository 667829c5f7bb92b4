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
extern "C" void plan(int bf16, int heads, int head_dim, int nseg, const int64_t* rows, const int* klen, int* tile,
                     int* size, int* chunks, int* item, int* row, int64_t* part) {
  const sphinx::Kv8Plan p = sphinx::plan_kv8(bf16 != 0, heads, head_dim, nseg, rows, klen);
  memcpy(size, p.size, 4 * nseg);
  *tile = p.tile;
  memcpy(chunks, p.chunks, 4 * nseg);
  memcpy(item, p.item, 4 * (nseg + 1));
  memcpy(row, p.row, 4 * (nseg + 1));
  memcpy(part, p.part, 8 * (nseg + 1));
}
extern "C" int64_t most(int heads, int nseg, const int64_t* rows, const int* klen) {
  return sphinx::kv8_most_parts(heads, nseg, rows, klen);
}
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


def plan(heads, rows, klen, bf16=True, head_dim=64):
    n = len(rows)
    rows, klen = np.ascontiguousarray(rows, np.int64), np.ascontiguousarray(klen, np.int32)
    tile = np.zeros(1, np.int32)
    out = [np.zeros(n, np.int32), np.zeros(n, np.int32), np.zeros(n + 1, np.int32), np.zeros(n + 1, np.int32), np.zeros(n + 1, np.int64)]
    lib().plan(int(bf16), heads, head_dim, n, ptr(rows), ptr(klen), ptr(tile), *(ptr(a) for a in out))
    return (int(tile[0]), *out)  # tile, size, chunks, item, row, part


def most(heads, rows, klen):
    return lib().most(heads, len(rows), ptr(np.ascontiguousarray(rows, np.int64)),
                      ptr(np.ascontiguousarray(klen, np.int32)))


@pytest.mark.parametrize("bf16,head_dim", [(True, 64), (True, 72), (False, 64)])
@pytest.mark.parametrize("seed", range(40))
def test_plan_covers_every_key_once_and_fits_its_workspace(seed, bf16, head_dim):
    rng = np.random.default_rng(seed)
    n = int(rng.integers(1, 65))
    heads = int(rng.choice([1, 2, 5, 16, 64]))
    rows = np.exp(rng.uniform(0, np.log(rng.choice([4, 200, 30000])), n)).astype(np.int64)
    cap = np.exp(rng.uniform(0, np.log(rng.choice([100, 30000, 4000000])), n)).astype(np.int64)
    bound = most(heads, rows, cap)
    for klen in (cap, (cap * rng.random(n)).astype(np.int64), cap * (rng.random(n) < 0.2)):
        tile, size, chunks, item, row, part = plan(heads, rows, klen, bf16, head_dim)
        blocks = (klen + 63) // 64
        assert (size >= 1).all() and (chunks >= 1).all() and tile in ((32, 128) if bf16 else (32,))
        # the last chunk of a segment holds a block, and the chunks together hold all of them
        assert (chunks * size >= blocks).all() and (((chunks - 1) * size < blocks) | (chunks == 1)).all()
        split = chunks > 1
        assert np.array_equal(np.diff(row), np.where(split, rows, 0)) and row[0] == 0
        assert np.array_equal(np.diff(part), np.where(split, rows * heads * chunks, 0)) and part[0] == 0
        assert np.array_equal(np.diff(item), (rows + tile - 1) // tile * chunks) and item[0] == 0
        assert part[-1] <= bound
        # a call is not cut finer than its purpose asks
        assert (np.diff(item) * heads)[split].sum() <= 1536


def test_rows_choose_the_tile():
    assert plan(4, [1], [9000])[0] == 32 and plan(4, [64], [9000])[0] == 32
    assert plan(4, [65], [9000])[0] == 128 and plan(4, [5000], [9000])[0] == 128
    assert plan(4, [5000], [9000], bf16=False)[0] == 32
    assert plan(4, [1] * 40 + [100], [9000] * 41)[0] == 32  # mostly single queries
    assert plan(4, [1] + [3000], [64, 9000])[0] == 128


def test_largest_calls_stay_in_range():
    rows = [(1 << 31) - 1]
    tile, size, chunks, item, row, part = plan(1, rows, [(1 << 31) - 1])
    assert chunks[0] == 1 and size[0] == 1 << 25 and item[1] == 1 << 24 and part[1] == 0
    tile, size, chunks, item, row, part = plan(1, [1], [(1 << 31) - 1])
    assert chunks[0] * int(size[0]) >= 1 << 25 and part[1] == chunks[0] <= most(1, [1], [(1 << 31) - 1])


@pytest.mark.parametrize("bf16,head_dim", [(True, 64), (True, 72), (False, 64)])
@pytest.mark.parametrize("seed", range(10))
def test_chunks_hold_more_than_half_of_the_least_limit(seed, bf16, head_dim):
    """More than half of four blocks, or of eight in 128-row tiles; and no more chunks than fours of blocks."""
    rng = np.random.default_rng(1000 + seed)
    n = int(rng.integers(1, 65))
    heads = int(rng.choice([1, 2, 8, 16]))
    rows = np.exp(rng.uniform(0, np.log(rng.choice([4, 300, 3000])), n)).astype(np.int64)
    klen = np.exp(rng.uniform(0, np.log(rng.choice([400, 3000, 1000000])), n)).astype(np.int64)
    for m in (n, 1, min(2, n)):
        tile, size, chunks, _, _, _ = plan(heads, rows[:m], klen[:m], bf16, head_dim)
        split = chunks > 1
        assert (size[split] >= (3 if tile == 32 else 5)).all()
        assert (chunks <= np.maximum(1, ((klen[:m] + 63) // 64 + 3) // 4)).all()


def test_the_chunks_that_the_limits_leave():
    assert plan(8, [1, 1], [33 * 64, 5 * 64])[1:3][0][1] == 3  # five blocks as three and two
    tile, size, *_ = plan(1, [300], [33 * 64])
    assert tile == 128 and size[0] == 7
