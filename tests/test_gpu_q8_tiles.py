"""Products of 8-bit matrices in every tile and form that they take, against 64 bits over the same bytes: sizes whose
plan (csrc/q8_rules.hpp, compiled for the host) is the tile that a test names."""
import numpy as np
import pytest

import q8_launch as L
from test_q8_plans import plan

torch = pytest.importorskip("torch")
S = pytest.importorskip("paper_2511_18672_amd")
B = S.binding

from test_gpu_q8 import GUARD, HALF, TYPE, U, dev, empty, numbers, pack, product  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda"
TILES = ["256x256", "192x256", "128x128", "128x64", "64x64", "few"]


def held(q, s, rows, cols):
    """The numbers that an 8-bit matrix holds, in 64 bits on the GPU."""
    wide = (cols + 127) // 128
    v = q[:rows * wide * 128].view(torch.float8_e4m3fn).float().double().view(rows, wide, 128)
    e = s[:rows * ((wide + 15) // 16 * 16)].view(rows, -1)[:, :wide].double() - 127
    return (v * torch.exp2(e)[:, :, None]).view(rows, -1)[:, :cols]


def operands(M, N, K):
    """Two matrices in 8 bits, their product and the sum of its terms' magnitudes in 64 bits."""
    a, b = pack(numbers(M, K, 1)), pack(numbers(N, K, 2) / np.sqrt(K))
    va, vb = held(*a, M, K), held(*b, N, K).T.contiguous()
    return a, b, va @ vb, va.abs() @ vb.abs()


def sum_error(K, size, bf16_cores=True):
    """K products one after the other at most, in groups of four or more, and on the 8-bit cores what eight products
    lose below 2^-13 of their largest: 8 2^-13 of it, so 2^-10 of their magnitudes."""
    return ((K / 4 + 8) * U + (2.0 ** -10 if bf16_cores else 0.0)) * size


def within(got, want, lost, half):
    """Each output is off by `lost` before its rounding, and by half a step."""
    err = (got.double() - want).abs()
    return bool((err <= lost + half * (want.abs() + lost) + 1e-38).all())


@pytest.mark.parametrize("kind, odt", [(L.BF16, "bf16"), (L.F32, "f32")])
@pytest.mark.parametrize("M, N, K", [(64, 64, 157 * 128), (70, 130, 40 * 128 - 3)])
def test_a_contraction_is_not_cut_without_a_workspace(kind, odt, M, N, K):
    """Sizes whose contraction is cut where there is one: the launcher takes none for it here."""
    assert plan(kind, False, M, N, (K + 127) // 128)[1] > 1
    a, b, c, size = operands(M, N, K)
    bias = dev(np.random.default_rng(3).normal(size=N))
    out = torch.full((M * N + 16,), GUARD, dtype=TYPE[odt][0], device=DEV)
    assert L.launch(B.lib(), kind, M, N, K, a, b, bias=bias, out=out, ldo=N,
                    stream=torch.cuda.current_stream().cuda_stream) == 0
    c = c + bias.double()
    assert within(out[:M * N].view(M, N), c, sum_error(K, size + c.abs(), odt == "bf16"), HALF[odt])
    assert (out[M * N:] == GUARD).all()
