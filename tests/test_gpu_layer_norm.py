"""The layer norm and its backward pass on the GPU against the 64-bit oracle."""
import numpy as np
import pytest

from oracle import q8 as Q

torch = pytest.importorskip("torch")
S = pytest.importorskip("paper_2511_18672_amd")
B = S.binding
pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPE = {"bf16": (torch.bfloat16, B.BF16), "f32": (torch.float32, B.F32)}
U = 2.0 ** -24                                # half a step of fp32
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}  # half a step of an output
GUARD = 7.0
# additions that follow each other in a sum over a row: up to 32 of a lane, then 4 + 2 between its lanes, 16 waves
DEPTH = 32 + 6 + 16


def dev(a, name="f32"):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(TYPE[name][0]).to(DEV)


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def strided(rows, ld, name, at=0):
    """A buffer of guard values for `rows` rows, and its view from element `at` (a multiple of 8)."""
    buf = torch.full((at + rows * ld + 5,), GUARD, dtype=TYPE[name][0], device=DEV)
    return buf, buf[at:]


def inputs(lens, cols, x, w, seed=0, offset=0.5):
    rng = np.random.default_rng([seed, cols, sum(lens)])
    rows, n = sum(lens), len(lens)
    return dict(x=dev(rng.normal(size=(rows, cols)) * np.exp(0.4 * rng.normal(size=cols)) + offset, x),
                w=dev(rng.normal(size=(n, cols)), w), b=dev(rng.normal(size=(n, cols)), w),
                dy=rng.normal(size=(rows, cols)), cu=np.concatenate([[0], np.cumsum(lens)]))


def norm_bounds(x, stats, w, b, y, cu, plus_one):
    """Largest errors of fp32 arithmetic: of the mean, of rstd (relative) and of y (before its rounding)."""
    mean = (DEPTH + 2) * U * np.abs(x).mean(axis=1, keepdims=True)
    # the variance is off by its sum, by the mean's error twice and by its square
    rel = (DEPTH + 8) * U + (mean * stats[:, 1:]) ** 2
    wr = np.repeat(np.abs(w) + (1.0 if plus_one else 0.0), np.diff(cu), axis=0)
    br = np.repeat(np.abs(b), np.diff(cu), axis=0)
    xh = np.abs((x - stats[:, :1]) * stats[:, 1:])
    return mean, rel, wr * (stats[:, 1:] * mean + xh * (rel + 6 * U)) + 4 * U * (np.abs(y) + br)


CASES = [([1], 1), ([1], 2), ([3], 5), ([1, 0, 4], 7), ([17], 8), ([9], 63), ([33], 64), ([20, 1], 127), ([130], 128),
         ([6], 129), ([0, 5, 0, 0, 3, 0], 333), ([13], 512), ([4, 4], 513), ([2], 1000), ([19], 1024), ([7], 1152),
         ([5], 1537), ([5], 2048), ([3], 2049), ([2, 1], 4099), ([3], 8192), ([2], 8193), ([2], 16384),
         ([1] * 64, 96), ([300, 5], 40)]


@pytest.mark.parametrize("lens, cols", CASES)
@pytest.mark.parametrize("x, w, y", [("f32", "f32", "bf16"), ("bf16", "f32", "f32"), ("f32", "bf16", "f32"),
                                     ("bf16", "bf16", "bf16")])
def test_forward(lens, cols, x, w, y):
    t, plus_one, eps = inputs(lens, cols, x, w), cols % 2 == 0, 1e-5
    rows, ldx, ldy = sum(lens), cols + 3, cols + 1
    _, xs = strided(rows, ldx, x, 8)
    buf, ys = strided(rows, ldy, y, 16)
    xs[:rows * ldx].view(rows, ldx)[:, :cols] = t["x"]
    stats = torch.full((rows, 2), GUARD, device=DEV)
    B.sphinx_layer_norm(TYPE[x][1], TYPE[w][1], TYPE[y][1], cols, eps, xs, ldx, t["w"], t["b"], cols, plus_one, t["cu"],
                        ys, ldy, stats)
    want, ws = Q.layer_norm(host(t["x"]), host(t["w"]), host(t["b"]), t["cu"], plus_one, eps)
    dm, dr, dy = norm_bounds(host(t["x"]), ws, host(t["w"]), host(t["b"]), want, t["cu"], plus_one)
    got = ys[:rows * ldy].view(rows, ldy)
    assert (np.abs(host(got[:, :cols]) - want) <= dy + HALF[y] * (np.abs(want) + dy) + 1e-37).all()
    assert (np.abs(host(stats[:, :1]) - ws[:, :1]) <= dm + U * np.abs(ws[:, :1])).all()
    assert (np.abs(host(stats[:, 1:]) - ws[:, 1:]) <= dr * ws[:, 1:]).all()
    assert (got[:, cols:] == GUARD).all() and (buf[:16] == GUARD).all() and (buf[16 + rows * ldy:] == GUARD).all()


def test_forward_without_weight_or_shift():
    for w, b in ((False, True), (True, False), (False, False)):
        t = inputs([5, 6], 200, "f32", "f32")
        for plus_one in (False, True):
            y = torch.empty(11, 200, device=DEV)
            B.sphinx_layer_norm(B.F32, B.F32, B.F32, 200, 1e-6, t["x"], 200, t["w"] if w else None,
                                t["b"] if b else None, 200, plus_one, t["cu"], y, 200)
            one = np.zeros((2, 200)) if plus_one else np.ones((2, 200))
            ww, bb = host(t["w"]) if w else one, host(t["b"]) if b else np.zeros((2, 200))
            want, ws = Q.layer_norm(host(t["x"]), ww, bb, t["cu"], plus_one, 1e-6)
            tol = norm_bounds(host(t["x"]), ws, ww, bb, want, t["cu"], plus_one)[2]
            assert (np.abs(host(y) - want) <= tol + U * np.abs(want)).all()


@pytest.mark.parametrize("cols", [5, 64, 128, 200, 1024, 5000])
def test_forward_rows_that_are_not_finite_or_alike(cols):
    t = inputs([6], cols, "f32", "f32")
    x = t["x"]
    x[1, cols // 2], x[3, 0], x[4] = float("nan"), float("inf"), 3.25
    y, stats = torch.empty_like(x), torch.empty(6, 2, device=DEV)
    B.sphinx_layer_norm(B.F32, B.F32, B.F32, cols, 1e-6, x, cols, t["w"], t["b"], cols, False, t["cu"], y, cols, stats)
    assert y[[1, 3]].isnan().all() and y[[0, 2, 5]].isfinite().all()
    # a constant row: its mean is exact up to the sum's roundings, and what is left is multiplied by at most 1000
    assert (y[4] - t["b"][0]).abs().max() <= 1000 * (DEPTH + 2) * U * 3.25 * t["w"].abs().max()


@pytest.mark.parametrize("lens, cols", CASES)
@pytest.mark.parametrize("x, y", [("f32", "f32"), ("bf16", "bf16")])
def test_forward_into_8_bits(lens, cols, x, y):
    t, rows = inputs(lens, cols, x, "f32"), sum(lens)
    (nq, ns), wide = B.sphinx_q8_bytes(rows, cols), (cols + 127) // 128
    q = torch.full((nq + 64,), 5, dtype=torch.uint8, device=DEV)
    s = torch.full((ns + 64,), 5, dtype=torch.uint8, device=DEV)
    stats = torch.empty(rows, 2, device=DEV)
    B.sphinx_layer_norm_q8(TYPE[x][1], B.F32, cols, 1e-6, t["x"], cols, t["w"], t["b"], cols, True, t["cu"], q, s, stats)
    assert (q[nq:] == 5).all() and (s[ns:] == 5).all()
    want, ws = Q.layer_norm(host(t["x"]), host(t["w"]), host(t["b"]), t["cu"], True, 1e-6)
    tol = norm_bounds(host(t["x"]), ws, host(t["w"]), host(t["b"]), want, t["cu"], True)[2]
    qv = q[:nq].view(torch.float8_e4m3fn).float().cpu().numpy().reshape(rows, wide * 128).astype(np.float64)
    assert (qv[:, cols:] == 0).all()
    e = s[:ns].view(rows, -1)[:, :wide].cpu().numpy().astype(np.int64) - 127
    e = np.repeat(e, 128, axis=1)[:, :cols]
    ref = Q.exponents(want)
    near = np.zeros_like(want, bool)  # groups whose largest number is within its error of a border between scales
    for j in range(0, cols, 128):
        top, lost = np.abs(want[:, j:j + 128]).max(axis=1), tol[:, j:j + 128].max(axis=1)
        border = 448.0 * np.ldexp(1.0, ref[:, j])
        near[:, j:j + 128] = (np.minimum(np.abs(top - border), np.abs(top - border / 2)) <= lost)[:, None]
    assert ((e == ref) | near).all() and (np.abs(e - ref) <= 1).all()
    # half a step of e4m3: 2^-4 of the number, 2^-10 of the unit for its subnormals
    got = qv[:, :cols] * np.ldexp(1.0, e)
    assert (np.abs(got - want) <= tol + 2.0 ** -4 * (np.abs(want) + tol) + np.ldexp(2.0 ** -10, e)).all()


# ---- backward ----------------------------------------------------------------
def run_backward(t, cols, x, w, g, plus_one, dx=True, dw=True, db=True, stream=None, ld=0):
    rows, n = t["x"].shape[0], len(t["cu"]) - 1
    ldg = cols + ld
    out = dict(dx=torch.full((rows, cols), GUARD, dtype=TYPE[g][0], device=DEV) if dx else None,
               dw=torch.full((n, ldg), GUARD, device=DEV) if dw else None,
               db=torch.full((n, ldg), GUARD, device=DEV) if db else None)
    ws = torch.full((B.sphinx_layer_norm_backward_workspace_bytes(cols, t["cu"]),), 255, dtype=torch.uint8, device=DEV)
    B.sphinx_layer_norm_backward(TYPE[x][1], TYPE[w][1], TYPE[g][1], cols, t["x"], cols, t["stats"], t["w"], cols,
                                 plus_one, t["cu"], t["g"], cols, out["dx"], cols, out["dw"], out["db"], ldg, ws, stream)
    return out


def with_stats(t, g):
    t["stats"] = dev(Q.layer_norm(host(t["x"]), None, None, t["cu"], False, 1e-5)[1])
    t["g"] = dev(t["dy"], g)
    return t


def check_backward(t, cols, g, plus_one, out):
    x, st, w, dy, cu = host(t["x"]), host(t["stats"]), host(t["w"]), host(t["g"]), t["cu"]
    want = Q.layer_norm_backward(x, st, w, cu, plus_one, dy)
    r = st[:, 1:]
    xh = np.abs((x - st[:, :1]) * r)
    gw = np.abs(dy) * np.repeat(np.abs(w) + (1.0 if plus_one else 0.0), np.diff(cu), axis=0)
    m1, m2 = gw.mean(axis=1, keepdims=True), (gw * xh).mean(axis=1, keepdims=True)
    # xh is off by 2 roundings, g by 2, each mean by its DEPTH additions and 5 more
    tol = r * U * ((DEPTH + 8) * (m1 + xh * m2) + 8 * (gw + m1 + 2 * xh * m2))
    got = host(out["dx"])
    assert (np.abs(got - want[0]) <= tol + HALF[g] * (np.abs(want[0]) + tol) + 1e-37).all()
    # a column's sum: at most a chunk's rows in turn, then 16 row groups, then a 16th of the chunks and 16 slices
    for name, ref, part in (("dw", want[1], np.abs(dy) * xh), ("db", want[2], np.abs(dy))):
        res = host(out[name])
        for i in range(len(cu) - 1):
            depth = (cu[i + 1] - cu[i]) / 16 + 64
            lim = U * (depth + 4) * part[cu[i]:cu[i + 1]].sum(axis=0)
            assert (np.abs(res[i, :cols] - ref[i]) <= lim + U * np.abs(ref[i])).all(), name
        assert (res[:, cols:] == GUARD).all()


@pytest.mark.parametrize("lens, cols", CASES + [([2000, 0, 700], 64), ([5000], 256), ([1200], 1152)])
@pytest.mark.parametrize("x, w, g", [("f32", "f32", "bf16"), ("bf16", "bf16", "bf16"), ("f32", "bf16", "f32"),
                                     ("bf16", "f32", "f32")])
def test_backward(lens, cols, x, w, g):
    t = with_stats(inputs(lens, cols, x, w), g)
    plus_one = cols % 2 == 1
    check_backward(t, cols, g, plus_one, run_backward(t, cols, x, w, g, plus_one, ld=3))


# around the limits of the calls whose columns are summed beside the rows: 32 to 1536 columns, 1024 rows of a segment,
# 12 MB of x and dy
@pytest.mark.parametrize("lens, cols", [([70], 31), ([70], 32), ([1024], 33), ([1025], 33), ([700, 0, 1024, 1], 32),
                                        ([1600], 100), ([1600, 3], 500), ([1700], 1000), ([1600], 1200), ([64], 1536),
                                        ([9] * 64, 95), ([1000, 0, 1000, 1000], 1200)])
@pytest.mark.parametrize("x, w, g", [("f32", "bf16", "f32"), ("bf16", "f32", "bf16")])
def test_backward_of_calls_small_and_not(lens, cols, x, w, g):
    t = with_stats(inputs(lens, cols, x, w), g)
    out = run_backward(t, cols, x, w, g, True, ld=5)
    check_backward(t, cols, g, True, out)
    # dx in the place of dy takes the sums from what dy held
    ws = torch.empty(B.sphinx_layer_norm_backward_workspace_bytes(cols, t["cu"]), dtype=torch.uint8, device=DEV)
    dw = torch.empty(len(lens), cols, device=DEV)
    B.sphinx_layer_norm_backward(TYPE[x][1], TYPE[w][1], TYPE[g][1], cols, t["x"], cols, t["stats"], t["w"], cols, True,
                                 t["cu"], t["g"], cols, t["g"], cols, dw, None, cols, ws)
    assert torch.equal(t["g"], out["dx"]) and torch.equal(dw, out["dw"][:, :cols])


def test_backward_outputs_left_out_and_calls_repeated():
    t = with_stats(inputs([700, 0, 41], 520, "bf16", "f32"), "bf16")
    full = run_backward(t, 520, "bf16", "f32", "bf16", True)
    for keep in ("dx", "dw", "db"):
        out = run_backward(t, 520, "bf16", "f32", "bf16", True, **{k: k == keep for k in ("dx", "dw", "db")})
        assert torch.equal(out[keep], full[keep])
    again = run_backward(t, 520, "bf16", "f32", "bf16", True)
    assert all(torch.equal(full[k], again[k]) for k in full)


def test_backward_of_no_rows_clears_the_sums():
    t = inputs([0, 0], 72, "f32", "f32")
    t.update(stats=torch.empty(0, 2, device=DEV), g=torch.empty(0, 72, device=DEV))
    out = run_backward(t, 72, "f32", "f32", "f32", False)
    assert (out["dw"] == 0).all() and (out["db"] == 0).all()


@pytest.mark.parametrize("cols", [40, 300, 4096])
def test_backward_keeps_what_is_not_finite_in_its_segment(cols):
    t = with_stats(inputs([37, 21, 30], cols, "f32", "f32"), "f32")
    ref = run_backward(t, cols, "f32", "f32", "f32", False)
    t["g"][40, 3] = float("nan")
    out = run_backward(t, cols, "f32", "f32", "f32", False)
    rows = torch.arange(88, device=DEV) != 40
    assert torch.equal(out["dx"][rows], ref["dx"][rows]) and out["dx"][40].isnan().all()
    for k in ("dw", "db"):
        assert torch.equal(out[k][[0, 2]], ref[k][[0, 2]]) and out[k][1, 3].isnan()
        keep = torch.arange(cols, device=DEV) != 3
        assert torch.equal(out[k][1][keep], ref[k][1][keep])


def test_a_stream_of_its_own_and_a_graph():
    t = with_stats(inputs([400, 90], 768, "f32", "f32"), "bf16")
    y = torch.empty(490, 768, dtype=torch.bfloat16, device=DEV)
    dx, dw, db = torch.empty_like(y), torch.empty(2, 768, device=DEV), torch.empty(2, 768, device=DEV)
    stats = torch.empty(490, 2, device=DEV)
    ws = torch.empty(B.sphinx_layer_norm_backward_workspace_bytes(768, t["cu"]), dtype=torch.uint8, device=DEV)

    def both(stream=None):
        B.sphinx_layer_norm(B.F32, B.F32, B.BF16, 768, 1e-6, t["x"], 768, t["w"], t["b"], 768, False, t["cu"], y, 768,
                            stats, stream)
        B.sphinx_layer_norm_backward(B.F32, B.F32, B.BF16, 768, t["x"], 768, stats, t["w"], 768, False, t["cu"], t["g"],
                                     768, dx, 768, dw, db, 768, ws, stream)

    outs = (y, stats, dx, dw, db)
    both()
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    for o in outs:
        o.zero_()
    side.wait_stream(torch.cuda.current_stream())
    both(side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for scale in (1.0, 0.5, 2.0):
        t["x"].mul_(scale)
        t["g"].mul_(scale)
        both()
        torch.cuda.synchronize()
        want = [o.clone() for o in outs]
        for o in outs:
            o.zero_()
        ws.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("cols", [40, 700, 1100, 3000, 9000])
@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_in_place(cols, name):
    """y in the place of x, dx in the place of dy."""
    t = with_stats(inputs([50, 0, 33], cols, name, "f32"), name)
    code = TYPE[name][1]
    ref = run_backward(t, cols, name, "f32", name, True)
    ws = torch.empty(B.sphinx_layer_norm_backward_workspace_bytes(cols, t["cu"]), dtype=torch.uint8, device=DEV)
    dw, db = torch.empty(3, cols, device=DEV), torch.empty(3, cols, device=DEV)
    B.sphinx_layer_norm_backward(code, B.F32, code, cols, t["x"], cols, t["stats"], t["w"], cols, True, t["cu"], t["g"],
                                 cols, t["g"], cols, dw, db, cols, ws)
    assert torch.equal(t["g"], ref["dx"]) and torch.equal(dw, ref["dw"]) and torch.equal(db, ref["db"])
    y = torch.empty_like(t["x"])
    args = (code, B.F32, code, cols, 1e-6, t["x"], cols, t["w"], t["b"], cols, False, t["cu"])
    B.sphinx_layer_norm(*args, y, cols)
    B.sphinx_layer_norm(*args, t["x"], cols)
    assert torch.equal(t["x"], y)


def test_offsets_past_32_bits():
    """More than 2^31 elements: the last rows are what they are in a call of their own."""
    rows, cols, last = 136000, 16384, 300
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    x.normal_(generator=torch.Generator(DEV).manual_seed(1))
    w = torch.rand(1, cols, device=DEV)
    y, q = torch.empty_like(x), torch.empty(rows * cols, dtype=torch.uint8, device=DEV)
    s = torch.empty(rows * cols // 128, dtype=torch.uint8, device=DEV)
    stats = torch.empty(rows, 2, device=DEV)
    few = [torch.empty(last, cols, dtype=torch.bfloat16, device=DEV), torch.empty(last, 2, device=DEV),
           torch.empty(last * cols, dtype=torch.uint8, device=DEV), torch.empty(last * cols // 128, dtype=torch.uint8,
                                                                                device=DEV)]
    call = (B.BF16, B.F32, B.BF16, cols, 1e-6)
    B.sphinx_layer_norm(*call, x, cols, w, None, cols, False, [0, rows], y, cols, stats)
    B.sphinx_layer_norm_q8(B.BF16, B.F32, cols, 1e-6, x, cols, w, None, cols, False, [0, rows], q, s)
    end = x[-last:].clone()
    B.sphinx_layer_norm(*call, end, cols, w, None, cols, False, [0, last], few[0], cols, few[1])
    B.sphinx_layer_norm_q8(B.BF16, B.F32, cols, 1e-6, end, cols, w, None, cols, False, [0, last], few[2], few[3])
    assert torch.equal(y[-last:], few[0]) and torch.equal(stats[-last:], few[1])
    assert torch.equal(q[-last * cols:], few[2]) and torch.equal(s[-last * cols // 128:], few[3])
    # backward, y as the gradient: two segments, of which the second is the last rows
    ws = torch.empty(B.sphinx_layer_norm_backward_workspace_bytes(cols, [0, rows - last, rows]), dtype=torch.uint8,
                     device=DEV)
    w2, dx = torch.cat([w, w]), torch.empty_like(x)
    B.sphinx_layer_norm_backward(B.BF16, B.F32, B.BF16, cols, x, cols, stats, w2, cols, False, [0, rows - last, rows], y,
                                 cols, dx, cols, None, None, cols, ws)
    B.sphinx_layer_norm_backward(B.BF16, B.F32, B.BF16, cols, end, cols, few[1], w, cols, False, [0, last], few[0], cols,
                                 few[0], cols, None, None, cols, None)
    assert torch.equal(dx[-last:], few[0])
