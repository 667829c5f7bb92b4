"""How a product of 8-bit matrices is divided (csrc/q8_rules.hpp), compiled for the host."""
import ctypes
import functools
import os
import subprocess
import tempfile

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include "q8_rules.hpp"
extern "C" void plan(int kind, int gelu, int M, int N, int KB, int* tile, int* pieces) {
  const sphinx::Q8Plan p = sphinx::plan_q8_matmul((sphinx::Q8Kind)kind, gelu != 0, M, N, KB);
  *tile = p.tile;
  *pieces = p.pieces;
}
"""
BF16, F32, GATED, BYTES = range(4)
TILES = [(256, 256), (192, 256), (128, 128), (128, 64), (64, 64), (16, 16)]


@functools.lru_cache(None)
def lib():
    with tempfile.TemporaryDirectory() as d:
        src, out = os.path.join(d, "rules.cpp"), os.path.join(d, "rules.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC",
                        "-I", os.path.join(ROOT, "paper_2511_18672_amd", "csrc"), src, "-o", out], check=True)
        return ctypes.CDLL(out)


def plan(kind, gelu, M, N, KB):
    t, p = ctypes.c_int(), ctypes.c_int()
    lib().plan(kind, int(gelu), M, N, KB, ctypes.byref(t), ctypes.byref(p))
    return TILES[t.value], p.value


@pytest.mark.parametrize("kind", [BF16, F32, GATED, BYTES])
def test_plans_hold(kind):
    rng = np.random.default_rng(1)
    for _ in range(4000):
        M, N = (int(np.exp(rng.uniform(0, np.log(1 << 18)))) for _ in range(2))
        KB = int(np.exp(rng.uniform(0, np.log(4000)))) - (rng.random() < 0.05)
        (rows, cols), pieces = plan(kind, rng.random() < 0.5, M, N, KB)
        assert pieces in (1, 2, 4, 8, 16) and (pieces == 1 or kind in (BF16, F32))
        if pieces > 1:  # every piece has blocks, and begins at a multiple of four
            per = ((KB + pieces - 1) // pieces + 3) // 4 * 4
            assert (pieces - 1) * per < KB <= pieces * per
        assert (rows == 16) == (kind in (BF16, F32) and M <= 16)
        assert kind != F32 or (rows, cols) != (256, 256)  # would spill
        assert kind != BYTES or cols >= 128  # whole blocks of the output's scales


def test_launches_stay_below_2_32_threads():
    for M, N in ((1 << 28, 1), (1 << 28, 128), (1, 1 << 28), (16, (1 << 28)), (1 << 20, 1 << 18), (1 << 23, 1 << 14)):
        for kind in (BF16, F32):
            for KB in (0, 1, 300):
                (rows, cols), pieces = plan(kind, False, M, N, KB)
                threads = 256 if rows * cols in (128 * 128, 128 * 64, 64 * 64) else 512
                n = -(-N // 16) if rows == 16 else -(-M // rows) * -(-N // cols)
                assert n * threads < 1 << 32 and pieces <= 16


def test_choices():
    """Measured choices: one round of the largest tiles that fill the CUs, small ones where few would be busy, cut
    contractions where even they are few."""
    assert plan(BF16, False, 32256, 1024, 32) == ((256, 256), 1)
    assert plan(BF16, False, 9677, 1024, 32) == ((192, 256), 1)
    assert plan(BF16, True, 9677, 4096, 8) == ((128, 128), 1)
    assert plan(BF16, False, 1333, 840, 9) == ((64, 64), 1)
    assert plan(F32, False, 4096, 1024, 76) == ((128, 128), 1)
    assert plan(BF16, False, 64, 64, 157)[1] > 1
