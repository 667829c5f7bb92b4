"""Sizes that do not fit the C interface are refused by the binding of the layer norm and the 8-bit matrices instead of
losing their high bits on the way.  No GPU is needed."""
import os

import pytest

torch = pytest.importorskip("torch")
S = pytest.importorskip("paper_2511_18672_amd")
B = S.binding

if not os.path.exists(B.LIB_PATH):
    pytest.skip("libsphinx.so not built", allow_module_level=True)

P32 = 1 << 32
f32, bf16, u8 = torch.float32, torch.bfloat16, torch.uint8


def meta(n, dtype):
    """A tensor of n elements without memory: these calls end before they look at one."""
    return torch.empty(n, dtype=dtype, device="meta")


def norm(cols=64, ldx=64, ldw=64, ldy=64, x=None, cu=(0, 2)):
    big = meta(abs(cols) * 2 + 64, bf16) if x is None else x
    B.sphinx_layer_norm(B.BF16, B.F32, B.BF16, cols, 1e-6, big, ldx, None, None, ldw, False, cu, meta(1 << 34, bf16), ldy)


def norm8(cols=64, ldx=64):
    B.sphinx_layer_norm_q8(B.BF16, B.F32, cols, 1e-6, meta(1 << 34, bf16), ldx, None, None, 64, False, (0, 2),
                           meta(1 << 34, u8), meta(1 << 34, u8))


def backward(cols=64, ldx=64, lddy=64, lddx=64, ldg=64):
    B.sphinx_layer_norm_backward(B.BF16, B.F32, B.BF16, cols, meta(1 << 34, bf16), ldx, meta(4, f32), None, 64, False,
                                 (0, 2), meta(1 << 34, bf16), lddy, meta(1 << 34, bf16), lddx, meta(1 << 34, f32), None, ldg,
                                 meta(1 << 34, u8))


def quantise(rows=4, cols=64, ldx=64):
    B.sphinx_q8_quantise(B.BF16, meta(1 << 40, bf16), ldx, rows, cols, False, meta(1 << 44, u8), meta(1 << 44, u8))


def matmul(M=4, N=4, K=64, ldo=4):
    m = meta(1 << 44, u8)
    B.sphinx_q8_matmul(B.BF16, M, N, K, m, m, m, m, B.F32, None, B.Q8_STORE, meta(1 << 44, bf16), ldo, None)


def matmul8(M=4, N=4, K=64):
    m = meta(1 << 44, u8)
    B.sphinx_q8_matmul_q8(M, N, K, m, m, m, m, B.F32, None, B.Q8_STORE, m, m)


@pytest.mark.parametrize("call, size", [(norm, "cols"), (norm8, "cols"), (backward, "cols"), (quantise, "rows"),
                                        (quantise, "cols"), (matmul, "M"), (matmul, "N"), (matmul, "K"), (matmul8, "M"),
                                        (matmul8, "N"), (matmul8, "K")])
@pytest.mark.parametrize("high", [P32, -P32])
def test_sizes_of_more_than_32_bits(call, size, high):
    with pytest.raises(ValueError, match="32 bits"):
        call(**{size: high + 64})


@pytest.mark.parametrize("call, ld", [(norm, "ldx"), (norm, "ldy"), (norm8, "ldx"), (backward, "ldx"), (backward, "lddy"),
                                      (backward, "lddx"), (quantise, "ldx"), (matmul, "ldo")])
@pytest.mark.parametrize("high", [1 << 64, -(1 << 64)])
def test_strides_of_more_than_64_bits(call, ld, high):
    with pytest.raises(ValueError):
        call(**{ld: high + 64})


def test_workspace_sizes():
    for cols in (P32 + 64, 64 - P32):
        with pytest.raises(ValueError, match="32 bits"):
            B.sphinx_layer_norm_backward_workspace_bytes(cols, (0, 2))


@pytest.mark.parametrize("mlp, fits", [(1 << 23, True), ((1 << 23) + 128, False), (1 << 26, False)])
def test_models_whose_rows_are_longer_than_an_8_bit_matrix_has(mlp, fits):
    """A product's tile addresses its rows with 32-bit offsets: matrices in 8 bits have at most 2^23 columns, those of a
    model as well."""
    import ctypes

    import workloads as W

    desc = B.model_desc(W.ModelCfg(D=128, heads=2, head_dim=64, mlp=mlp, L=1, dtype="bf16"), 1 << 20)
    reqs = B.make_requests([W.Request(1, 4, 4)])
    calls = [lambda: B.sphinx_model_q8_bytes(desc), lambda: B.sphinx_refine_q8_workspace_bytes(desc, reqs, 4)]
    for call in calls:
        if fits:
            assert call() > 0
        else:
            with pytest.raises(S.SphinxError, match="UNSUPPORTED"):
                call()
    pack = B.lib().sphinx_model_q8_pack(ctypes.byref(desc), 1 << 20, 0, None)
    assert B.STATUS_NAMES[pack] == ("SPHINX_E_WORKSPACE" if fits else "SPHINX_E_UNSUPPORTED")
