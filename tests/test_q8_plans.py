"""Products that have no workspace, as the refinement step's, are not cut (csrc/q8_rules.hpp, compiled for the host)."""
import ctypes
import functools
import os
import shutil
import subprocess
import tempfile

import numpy as np
import pytest

import q8_launch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include "q8_rules.hpp"
extern "C" int plan(int kind, int gelu, int M, int N, int KB, int whole) {
  const sphinx::Q8Plan p = sphinx::plan_q8_matmul((sphinx::Q8Kind)kind, gelu != 0, M, N, KB, whole != 0);
  return p.tile * 100 + p.pieces;
}
extern "C" int has(int kind, int tile) { return sphinx::q8_has_tile((sphinx::Q8Kind)kind, (sphinx::Q8Tile)tile); }
// Row counts up to `rows` at which the plan with a workspace is another one than without.
extern "C" int differing(int kind, int gelu, int rows, int N, int KB) {
  int n = 0;
  for (int M = 1; M <= rows; M += M < 1000 ? 1 : 37) n += plan(kind, gelu, M, N, KB, 0) != plan(kind, gelu, M, N, KB, 1);
  return n;
}
"""
BF16, F32, GATED, BYTES = range(4)


@functools.lru_cache(None)
def lib():
    with tempfile.TemporaryDirectory() as d:
        src, out = os.path.join(d, "plans.cpp"), os.path.join(d, "plans.so")
        with open(src, "w") as f:
            f.write(SOURCE)
        subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC",
                        "-I", os.path.join(ROOT, "paper_2511_18672_amd", "csrc"), src, "-o", out], check=True)
        return ctypes.CDLL(out)


def plan(kind, gelu, M, N, KB, whole=False):
    """(tile, pieces)"""
    return divmod(lib().plan(kind, int(gelu), M, N, KB, int(whole)), 100)


@pytest.mark.parametrize("kind", [BF16, F32, GATED, BYTES])
def test_no_pieces_without_a_workspace(kind):
    rng = np.random.default_rng(1)
    cut = 0
    for _ in range(4000):
        M, N, KB = (int(np.exp(rng.uniform(0, np.log(hi)))) for hi in (1 << 17, 1 << 14, 4000))
        gelu = rng.random() < 0.5
        free = plan(kind, gelu, M, N, KB)
        tile, pieces = plan(kind, gelu, M, N, KB, True)
        assert pieces == 1
        assert free[1] > 1 or free[0] == tile  # the same tile, where the contraction would not have been cut
        cut += free[1] > 1
    assert (cut > 100) == (kind in (BF16, F32))


def test_plans_name_tiles_that_the_launcher_has():
    rng = np.random.default_rng(2)
    have = {kind: {t for t in range(6) if lib().has(kind, t)} for kind in range(4)}
    assert have == {BF16: {0, 1, 2, 3, 4, 5}, F32: {1, 2, 3, 4, 5}, GATED: {0, 1, 2, 3, 4}, BYTES: {0, 1, 2}}
    for kind in have:
        seen = set()
        for _ in range(4000):
            M, N, KB = (int(np.exp(rng.uniform(0, np.log(hi)))) for hi in (1 << 18, 1 << 14, 4000))
            seen.add(plan(kind, rng.random() < 0.5, M, N, KB, rng.random() < 0.5)[0])
        assert seen == have[kind]


def test_the_refinement_steps_products_lose_nothing_by_it():
    """Models of D = 128 to 2048: the QKV product is planned alike with and without a workspace."""
    for D in range(128, 2049, 128):
        assert lib().differing(BF16, 0, 80000, 3 * D, D // 128) == 0, D


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"),
                    reason="hipcc not available")
def test_structures_of_the_launcher_are_the_tests_own(tmp_path):
    src = tmp_path / "layout.hip"
    src.write_text(q8_launch.layout_checks())
    cmd = [shutil.which("hipcc") or "/opt/rocm/bin/hipcc", "--offload-arch=gfx950", "--cuda-host-only", "-std=c++17",
           "-fsyntax-only", "-I", os.path.join(ROOT, "include"), "-I",
           os.path.join(ROOT, "paper_2511_18672_amd", "csrc"), str(src)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def test_the_launcher_refuses_scaled_columns_that_end_inside_32():
    """A tile's epilogue scales 32 columns or none.  Refused before any HIP call."""
    S = pytest.importorskip("paper_2511_18672_amd")
    if not os.path.exists(S.binding.LIB_PATH):
        pytest.skip("libsphinx.so not built")
    call = lambda kind=q8_launch.BF16, **e: q8_launch.launch(  # noqa: E731
        S.lib(), kind, 100, 96, 64, (1 << 20, 1 << 20), (1 << 20, 1 << 20), out=1 << 20, ldo=96, qscale=0.5, **e)
    invalid = 1  # hipErrorInvalidValue
    assert call(qcols=8) == invalid and call(qcols=40) == invalid
    assert call(qcols=32, epi=q8_launch.GELU) == invalid and call(q8_launch.F32, qcols=32) == invalid
