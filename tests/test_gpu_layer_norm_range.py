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


def far_rows(lens, cols, name):
    """Rows of finite numbers whose sum or sum of squares passes fp32's largest, ordinary ones between them."""
    t = inputs(lens, cols, "f32", "f32")
    x, rng = host(t["x"]), np.random.default_rng(cols)
    g = rng.normal(size=cols)
    x[0] = np.ldexp(g, 80)                                 # squares past it, 2^70 and more of them
    x[1] = np.ldexp(np.clip(g, -3, 3), 124)                # and its variance past it in any unit
    x[2] = 2.0 ** 120                                      # a constant, whose sum passes it from 256 columns on
    x[3] = np.where(np.arange(cols) % 2 == 0, 1.5, 1.0) * 2.0 ** 124  # sum and squares
    x[5] = 1.0
    x[5, cols // 2] = -(2.0 ** 125)                        # one far number beside small ones
    x[6] = np.ldexp(g + 0.5, 63)                           # at the edge
    t["x"] = dev(x, name)
    return t


def far_bounds(x, st, w, b, y, plus_one):
    """test_gpu_layer_norm's bounds where the variance is far above eps."""
    from test_gpu_layer_norm import DEPTH

    # the mean is off by its sum's roundings, as a part of the deviation
    mean = (DEPTH + 3) * U * np.abs(x).mean(axis=1, keepdims=True) * st[:, 1:]
    rel = (DEPTH + 8) * U + mean ** 2
    xh, wr = np.abs((x - st[:, :1]) * st[:, 1:]), np.abs(w) + (1.0 if plus_one else 0.0)
    return wr * (mean + xh * (rel + 6 * U)) + 4 * U * (np.abs(y) + np.abs(b))


@pytest.mark.parametrize("cols", [16, 40, 333, 700, 1024, 1100, 1536, 2000, 3000, 5000, 9000, 16384])
@pytest.mark.parametrize("x, y", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16")])
def test_forward_of_rows_that_pass_fp32_on_the_way(cols, x, y):
    from test_gpu_layer_norm import DEPTH, HALF

    t = far_rows([8], cols, x)
    rows, code = 8, TYPE[y][1]
    out, stats = torch.empty(rows, cols, dtype=TYPE[y][0], device=DEV), torch.empty(rows, 2, device=DEV)
    args = (cols, 1e-6, t["x"], cols, t["w"], t["b"], cols, False, t["cu"])
    B.sphinx_layer_norm(TYPE[x][1], B.F32, code, *args, out, cols, stats)
    xs, w, b = host(t["x"]), host(t["w"]), host(t["b"])
    want, st = Q.layer_norm(xs, w, b, t["cu"], False, 1e-6)
    got, kept = host(out), host(stats)
    assert np.isfinite(got).all() and np.isfinite(kept).all()
    far = np.array([0, 1, 3, 4, 5, 6, 7])  # all but the constant row
    lost = far_bounds(xs, st, w, b, want, False)
    assert (np.abs(got - want) <= lost + HALF[y] * (np.abs(want) + lost) + 1e-37)[far].all()
    assert (got[2] == host(dev(b, y))[0]).all() if y == "bf16" else (got[2] == b[0]).all()
    assert (np.abs(kept[:, 0] - st[:, 0]) <= (DEPTH + 3) * U * np.abs(xs).mean(axis=1) + U * np.abs(st[:, 0])).all()
    # 1 / deviations below 2^-126 are kept in steps of 2^-149
    rel = (DEPTH + 8) * U + ((DEPTH + 3) * U * np.abs(xs).mean(axis=1) * st[:, 1]) ** 2
    assert (np.abs(kept[:, 1] - st[:, 1]) <= rel * st[:, 1] + 2.0 ** -149)[far].all()
    assert kept[2, 0] == 2.0 ** 120 and abs(kept[2, 1] - 1000.0) < 0.001
    # into 8 bits: as the fp32 output quantised, number for number
    wide = (cols + 127) // 128
    q, s = (torch.zeros(n, dtype=torch.uint8, device=DEV) for n in B.sphinx_q8_bytes(rows, cols))
    B.sphinx_layer_norm_q8(TYPE[x][1], B.F32, *args, q, s)
    full = torch.empty(rows, cols, device=DEV)
    B.sphinx_layer_norm(TYPE[x][1], B.F32, B.F32, *args, full, cols)
    e = np.repeat(s.view(rows, -1)[:, :wide].cpu().numpy().astype(np.int64) - 127, 128, axis=1)
    v = q.view(torch.float8_e4m3fn).float().cpu().numpy().reshape(rows, -1).astype(np.float64) * np.ldexp(1.0, e)
    assert np.array_equal(v[:, :cols], Q.quantise(host(full)))
    if x == y:  # in place
        B.sphinx_layer_norm(code, B.F32, code, *args, t["x"], cols)
        assert torch.equal(t["x"], out)


@pytest.mark.parametrize("cols", [40, 333, 1024, 3000, 9000])
def test_rows_beside_far_and_infinite_ones_are_as_they_are_alone(cols):
    t = far_rows([8], cols, "f32")
    t["x"][1, 3], t["x"][3, cols - 1], t["x"][5, 0] = float("inf"), float("nan"), -float("inf")
    args = (t["w"], t["b"], cols, False)
    y = torch.empty(8, cols, device=DEV)
    B.sphinx_layer_norm(B.F32, B.F32, B.F32, cols, 1e-6, t["x"], cols, *args, [0, 8], y, cols)
    assert y[[1, 3, 5]].isnan().all() and y[[0, 2, 4, 6, 7]].isfinite().all()
    for i in (0, 2, 4, 6, 7):
        one = torch.empty(1, cols, device=DEV)
        B.sphinx_layer_norm(B.F32, B.F32, B.F32, cols, 1e-6, t["x"][i].clone(), cols, *args, [0, 1], one, cols)
        assert torch.equal(one[0], y[i])


@pytest.mark.parametrize("lens, cols", [([6, 5], 40), ([1030], 40), ([6, 5], 1000), ([9], 1100), ([1030], 1100), ([7], 3000),
                                        ([5, 2], 9000)])
@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_backward_of_far_rows(lens, cols, name):
    """Numbers up to 2^126, whose deviations' reciprocals are at the low end of fp32."""
    t, rng = inputs(lens, cols, name, "f32"), np.random.default_rng(cols)
    t["x"][::2] = dev(np.ldexp(np.clip(rng.normal(size=t["x"][::2].shape), -3.9, 3.9), 124), name)
    t["x"][1] = dev(np.ldexp(rng.normal(size=cols), 70), name)
    t["dy"] = np.ldexp(t["dy"], 30)  # so that dx is far from fp32's low end
    t = with_stats(t, "f32")
    check_backward(t, cols, "f32", False, run_backward(t, cols, name, "f32", "f32", False, ld=3))
