"""bench.py prices each product at the peak of the type that it runs in."""
import pytest

bench = pytest.importorskip("bench")


def test_a_step_is_priced_at_the_peaks_of_its_types():
    flop = {"gemm_qkv": 3e12, "gemm_out": 1e12, "gemm_mlp1": 4e12, "gemm_mlp2": 5e12}
    assert bench.mfma_seconds(2, 7e12, flop, "model") == pytest.approx(2 * 20e12 / 2.5e15)
    # attention and the output projection stay in bf16
    assert bench.mfma_seconds(2, 7e12, flop, "fp8") == pytest.approx(2 * (8e12 / 2.5e15 + 12e12 / 5e15))
