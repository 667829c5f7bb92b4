"""Rows of the layer norm near the ends of fp32's range, forward and backward, against the 64-bit oracle: whatever is
finite stays finite."""
import numpy as np
import pytest

from oracle import q8 as Q

torch = pytest.importorskip("torch")
S = pytest.importorskip("paper_2511_18672_amd")
B = S.binding

from test_gpu_layer_norm import TYPE, U, check_backward, dev, host, inputs, run_backward, with_stats  # noqa: E402

pytestmark = pytest.mark.gpu

DEV = "cuda"


# Widths that leave lanes behind the last column (and 1024, which leaves none), for each number of lanes of a row; rows
# enough in one segment for sums in a launch of their own, and few enough for sums beside the rows.
@pytest.mark.parametrize("lens, cols", [([5], 20), ([1030], 20), ([9, 0, 4], 40), ([1030], 40), ([7, 3], 333),
                                        ([1030, 2], 333), ([7, 3], 1000), ([7, 3], 1024), ([7], 1100), ([1030], 1100),
                                        ([7, 3], 2000), ([5], 3000), ([5], 5000), ([4, 1], 9000)])
@pytest.mark.parametrize("x, g", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
def test_backward_of_a_constant_row_of_a_large_number(lens, cols, x, g):
    """mean * rstd passes fp32's largest, though x - mean is zero in every column."""
    t = inputs(lens, cols, x, "f32")
    t["x"][1], t["x"][sum(lens) - 1] = 2.0 ** 119, -(2.0 ** 125)
    t = with_stats(t, g)
    assert float(t["stats"][1, 0]) == 2.0 ** 119 and float(t["stats"][1, 1]) > 300.0
    for keep in (dict(), dict(dw=False, db=False)):
        out = run_backward(t, cols, x, "f32", g, True, ld=3, **keep)
        assert out["dx"].isfinite().all()
        if not keep:
            check_backward(t, cols, g, True, out)
