"""Matrices in 8 bits with a scale for each block of 128 and their products, against the 64-bit oracle."""
import numpy as np
import pytest

from oracle import q8 as Q

torch = pytest.importorskip("torch")
S = pytest.importorskip("paper_2511_18672_amd")
B = S.binding
pytestmark = pytest.mark.gpu

DEV = "cuda"
TYPE = {"bf16": (torch.bfloat16, B.BF16), "f32": (torch.float32, B.F32)}
U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
GUARD = 7.0


def dev(a, name="f32"):
    return torch.from_numpy(np.ascontiguousarray(a, np.float32)).to(TYPE[name][0]).to(DEV)


def host(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def values(q, s, rows, cols):
    """The numbers that an 8-bit matrix holds, and the check of its padding."""
    wide = (cols + 127) // 128
    v = q[:rows * wide * 128].view(torch.float8_e4m3fn).float().cpu().numpy().astype(np.float64).reshape(rows, wide * 128)
    assert (v[:, cols:] == 0).all()
    e = s[:rows * ((wide + 15) // 16 * 16)].view(rows, -1)[:, :wide].cpu().numpy().astype(np.int64) - 127
    return (v * np.ldexp(1.0, np.repeat(e, 128, axis=1)))[:, :cols]


def empty(rows, cols, extra=32):
    return [torch.full((n + extra,), 5, dtype=torch.uint8, device=DEV) for n in B.sphinx_q8_bytes(rows, cols)]


def pack(x, name="f32", square=False):
    """An 8-bit matrix from host numbers."""
    rows, cols = x.shape
    t = dev(x, name)
    q, s = empty(rows, cols)
    B.sphinx_q8_quantise(TYPE[name][1], t, cols, rows, cols, square, q, s)
    return q, s


def numbers(rows, cols, seed=0):
    rng = np.random.default_rng([seed, rows, cols])
    return rng.normal(size=(rows, cols)) * np.exp(1.5 * rng.normal(size=(rows, 1)) + rng.normal(size=cols))


SIZES = [(1, 1), (1, 128), (3, 129), (128, 128), (127, 7), (129, 300), (37, 513), (300, 64), (260, 1025), (5, 4000)]


@pytest.mark.parametrize("rows, cols", SIZES)
@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("square", [False, True])
def test_quantise(rows, cols, name, square):
    x, ld = numbers(rows, cols), cols + 5
    x[rows // 2, : cols // 2] = 0.0
    if rows > 2 and cols > 3:
        x[0, 0], x[1, 2], x[rows - 1, cols - 1] = np.nan, np.inf, -np.inf
    buf = torch.full((rows, ld), GUARD, dtype=TYPE[name][0], device=DEV)
    buf[:, :cols] = dev(x, name)
    x = host(buf[:, :cols])
    q, s = empty(rows, cols)
    qt, st = empty(cols, rows)
    sums = torch.full((cols + 3,), GUARD, device=DEV)
    ws = torch.full((B.sphinx_q8_quantise_workspace_bytes(rows, cols),), 255, dtype=torch.uint8, device=DEV)
    B.sphinx_q8_quantise(TYPE[name][1], buf, ld, rows, cols, square, q, s, qt, st, sums, ws)
    want = Q.quantise(x, square)
    assert np.array_equal(values(q, s, rows, cols), want, equal_nan=True)
    wt = want.T if square else Q.quantise(x.T)
    assert np.array_equal(values(qt, st, cols, rows), wt, equal_nan=True)
    for t, n in zip((q, s, qt, st), B.sphinx_q8_bytes(rows, cols) + B.sphinx_q8_bytes(cols, rows)):
        assert (t[n:] == 5).all()
    ok = np.isfinite(x).all(axis=0)  # 8 rows of a thread, 16 groups, then a 16th of the tiles and 16 slices
    lim = U * (8 + 16 + rows / 2048 + 17) * np.abs(x[:, ok]).sum(axis=0)
    assert (np.abs(host(sums)[:cols][ok] - x[:, ok].sum(axis=0)) <= lim).all()
    assert not np.isfinite(host(sums)[:cols][~ok]).any() and (sums[cols:] == GUARD).all()
    # one output at a time, the same bits
    for keep in ((q, s, None, None), (None, None, qt, st)):
        new = [None if t is None else torch.full_like(t, 5) for t in keep]
        B.sphinx_q8_quantise(TYPE[name][1], buf, ld, rows, cols, square, *new)
        for k, (a, b) in enumerate(zip(new, keep)):
            if a is not None and k % 2 == 0:
                assert torch.equal(a, b)
        r, c = (rows, cols) if keep[0] is not None else (cols, rows)
        a, b = [t for t in new if t is not None], [t for t in keep if t is not None]
        assert np.array_equal(values(*a, r, c), values(*b, r, c), equal_nan=True)


# around the limits of the inputs whose columns are summed beside the tiles: 129 to 2048 rows, 32 columns, 8 MB
@pytest.mark.parametrize("rows, cols", [(129, 31), (129, 32), (129, 33), (2048, 40), (2049, 40), (1024, 2048),
                                        (1025, 2048), (1025, 4096)])
@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_column_sums_of_inputs_small_and_not(rows, cols, name):
    buf = torch.full((rows, cols + 3), GUARD, dtype=TYPE[name][0], device=DEV)
    buf[:, :cols] = dev(numbers(rows, cols), name)
    x = host(buf[:, :cols])
    ws = torch.full((B.sphinx_q8_quantise_workspace_bytes(rows, cols),), 255, dtype=torch.uint8, device=DEV)
    # 16 rows of a thread, 8 slices and 16 groups of them, or what test_quantise counts
    lim = U * (8 + 16 + rows / 128 + 17) * np.abs(x).sum(axis=0)
    for square in (False, True):
        sums = torch.full((cols + 3,), GUARD, device=DEV)
        q, s = empty(rows, cols)
        B.sphinx_q8_quantise(TYPE[name][1], buf, cols + 3, rows, cols, square, q, s, None, None, sums, ws)
        assert (np.abs(host(sums)[:cols] - x.sum(axis=0)) <= lim).all() and (sums[cols:] == GUARD).all()
        alone = torch.empty(cols, device=DEV)
        B.sphinx_q8_quantise(TYPE[name][1], buf, cols + 3, rows, cols, square, None, None, None, None, alone, ws)
        assert torch.equal(alone, sums[:cols])


def test_quantise_extreme_numbers():
    x = np.zeros((6, 128), np.float32)
    x[0, :4] = 3e38, -3.3e38, 1e38, 1.0     # past 448 2^119: saturates
    x[1, :3] = 2.0 ** -126, -2.0 ** -120, 2.0 ** -140
    x[2, :2] = 448.0, 0.4375 * 2 ** -6
    x[3, :2] = 448.0000305, 1.0
    x[4, :2] = 2.0 ** -149, 0.0
    x[5] = np.inf
    q, s = empty(6, 128)
    B.sphinx_q8_quantise(B.F32, torch.from_numpy(x).to(DEV), 128, 6, 128, False, q, s)
    assert np.array_equal(values(q, s, 6, 128), Q.quantise(x.astype(np.float64)), equal_nan=True)
    assert s[:96].view(6, 16)[:, 0].cpu().tolist() == [246, 27, 127, 128, 27, 27]


def test_quantise_rounds_ties_to_even():
    grid = np.array([8 * (1 + k / 16) for k in range(16)] + [2.0 ** -9 * (k + 0.5) for k in range(8)])
    x = np.concatenate([[448.0], grid, -grid])[None]
    assert np.array_equal(values(*pack(x), 1, x.shape[1]), Q.quantise(x))


def test_sums_of_no_rows():
    sums = torch.full((9,), GUARD, device=DEV)
    B.sphinx_q8_quantise(B.F32, torch.empty(0, 9, device=DEV), 9, 0, 9, False, None, None, None, None, sums,
                         torch.empty(0, dtype=torch.uint8, device=DEV))
    assert (sums == 0).all()


# ---- products ------------------------------------------------------------------
def product(odt, a, b, M, N, K, bias=None, bdt="f32", epilogue=B.Q8_STORE, before=None, ld=0, stream=None):
    ldo = N + ld
    buf = torch.full((M * ldo + 16,), GUARD, dtype=TYPE[odt][0], device=DEV)
    out = buf[:M * ldo].view(M, ldo)
    if before is not None:
        out[:, :N] = before
    ws = torch.full((B.sphinx_q8_matmul_workspace_bytes(TYPE[odt][1], M, N, K),), 255, dtype=torch.uint8, device=DEV)
    B.sphinx_q8_matmul(TYPE[odt][1], M, N, K, *a, *b, TYPE[bdt][1], bias, epilogue, buf, ldo, ws, stream)
    assert (out[:, N:] == GUARD).all() and (buf[M * ldo:] == GUARD).all()
    return out[:, :N]


def tolerance(odt, c, size, K):
    """Roundings of the sums (K products one after the other at most, in groups of four or more) and, with bf16
    outputs, what eight products lose below 2^-13 of their largest: 8 2^-13 of it, so 2^-10 of their magnitudes."""
    tol = (K / 4 + 8) * U * size + (2.0 ** -10 * size if odt == "bf16" else 0.0)
    return tol + HALF[odt] * (np.abs(c) + tol) + 1e-38


SHAPES = [(1, 1, 1), (1, 8, 128), (2, 100, 7), (5, 131, 300), (16, 64, 1024), (17, 257, 129), (33, 31, 640), (64, 128, 128),
          (65, 200, 1333), (128, 128, 256), (129, 127, 385), (200, 384, 512), (300, 264, 1000), (513, 70, 2050),
          (640, 520, 140), (40, 1030, 900), (1100, 16, 257), (96, 96, 9000), (257, 513, 4224),
          (1, 4096, 1024), (3, 40, 9000), (20, 33, 1100), (32, 100, 5000), (31, 15, 200)]


@pytest.mark.parametrize("M, N, K", SHAPES)
@pytest.mark.parametrize("odt", ["f32", "bf16"])
def test_product(M, N, K, odt):
    xa, xb = numbers(M, K, 1), numbers(N, K, 2) / np.sqrt(K)
    a, b = pack(xa), pack(xb, square=N % 2 == 0)
    va, vb = values(*a, M, K), values(*b, N, K)
    rng = np.random.default_rng(3)
    for bdt in ("f32", "bf16", None):
        bias = None if bdt is None else dev(rng.normal(size=N), bdt)
        c, size = Q.matmul(va, vb, None if bias is None else host(bias))
        tol = tolerance(odt, c, size + np.abs(c), K)
        ld = 0 if bdt is None else 3 if bdt == "f32" else 8
        got = host(product(odt, a, b, M, N, K, bias, bdt or "f32", ld=ld))
        assert (np.abs(got - c) <= tol).all(), np.abs(got - c).max()
    # GELU has a slope of at most 1.13; its own arithmetic adds 16 roundings of z and its result
    g = Q.gelu(c)
    tol0 = 1.13 * tolerance("f32", c, size, K) + 16 * U * (np.abs(c) + 1) + (1.13 * 2.0 ** -10 * size if odt == "bf16" else 0)
    got = host(product(odt, a, b, M, N, K, epilogue=B.Q8_GELU))
    assert (np.abs(got - g) <= tol0 + HALF[odt] * (np.abs(g) + tol0)).all()
    before = dev(rng.normal(size=(M, N)), odt)
    total = c + host(before)
    tol1 = tolerance(odt, total, size + np.abs(total), K)
    assert (np.abs(host(product(odt, a, b, M, N, K, epilogue=B.Q8_ADD, before=before, ld=1)) - total) <= tol1).all()


@pytest.mark.parametrize("odt", ["f32", "bf16"])
def test_tiles_of_every_size_add_up_alike(odt):
    """Products of more than 16 rows whose contraction is not cut give the same bits for a row whatever the rows and
    columns beside it, so whatever the tile (64x64 to 256x256)."""
    M, N, K = 9000, 2304, 300
    a, b = pack(numbers(M, K, 1)), pack(numbers(N, K, 2))
    full = product(odt, a, b, M, N, K)
    for m, n in ((17, 2304), (70, 64), (400, 2304), (1500, 1000), (9000, 200), (4000, 2304)):
        assert torch.equal(product(odt, a, b, m, n, K), full[:m, :n]), (m, n)


def test_product_without_a_contraction_is_the_bias():
    u8 = torch.empty(0, dtype=torch.uint8, device=DEV)
    bias = dev(np.arange(70.0))
    for odt in ("f32", "bf16"):
        for M in (1, 40, 150):
            got = product(odt, (u8, u8), (u8, u8), M, 70, 0, bias)
            assert torch.equal(got, bias.to(TYPE[odt][0]).expand(M, 70))


def test_product_with_scales_far_apart():
    """Blocks of one row with exponents from -100 to 100: a wrong scale or block would be off by far."""
    M, N, K = 70, 90, 1400
    rng = np.random.default_rng(5)
    xa, xb = rng.normal(size=(M, K)), rng.normal(size=(N, K))
    for k in range(0, K, 128):
        e = rng.integers(-50, 51, size=(M, 1))
        xa[:, k:k + 128] = np.ldexp(xa[:, k:k + 128], e)
        xb[:, k:k + 128] = np.ldexp(xb[:, k:k + 128], rng.integers(-8, 9, size=(N, 1)))
    a, b = pack(xa), pack(xb)
    for odt in ("f32", "bf16"):
        c, size = Q.matmul(values(*a, M, K), values(*b, N, K))
        assert (np.abs(host(product(odt, a, b, M, N, K)) - c) <= tolerance(odt, c, size, K)).all()


@pytest.mark.parametrize("M, N, K", [(3, 40, 300), (200, 150, 700), (40, 300, 4000)])
@pytest.mark.parametrize("odt", ["f32", "bf16"])
def test_product_keeps_nan_in_its_row_and_column(M, N, K, odt):
    xa, xb = numbers(M, K, 7), numbers(N, K, 8)
    ref = product(odt, pack(xa), pack(xb), M, N, K)
    xa[1, K - 1], xb[N - 1, 5] = np.nan, np.inf
    got = product(odt, pack(xa), pack(xb), M, N, K)
    hit = torch.zeros(M, N, dtype=torch.bool, device=DEV)
    hit[1], hit[:, N - 1] = True, True
    assert got[hit].isnan().all() and torch.equal(got[~hit], ref[~hit])


@pytest.mark.parametrize("odt", ["f32", "bf16"])
def test_product_repeats_on_streams_and_in_graphs(odt):
    for M, N, K in ((3, 700, 1500), (300, 260, 900), (130, 140, 8000)):
        a, b = pack(numbers(M, K, 1)), pack(numbers(N, K, 2))
        want = product(odt, a, b, M, N, K)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            got = product(odt, a, b, M, N, K)
        side.synchronize()
        assert torch.equal(got, want)
        out = torch.empty(M, N, dtype=TYPE[odt][0], device=DEV)
        x = dev(numbers(M, K, 1))
        ws = torch.empty(B.sphinx_q8_matmul_workspace_bytes(TYPE[odt][1], M, N, K), dtype=torch.uint8, device=DEV)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            B.sphinx_q8_quantise(B.F32, x, K, M, K, False, *a)
            B.sphinx_q8_matmul(TYPE[odt][1], M, N, K, *a, *b, B.F32, None, B.Q8_STORE, out, N, ws)
        for scale in (1.0, 3.0, 0.25):
            x.mul_(scale)
            out.fill_(GUARD)
            ws.fill_(200)
            graph.replay()
            torch.cuda.synchronize()
            got = out.clone()
            assert torch.equal(got, product(odt, pack(host(x)), b, M, N, K))


def test_offsets_past_32_bits():
    """Matrices of more than 2^32 bytes: their last rows and columns are what they are in a call of their own."""
    M, K, N, last = 131072 + 700, 33000, 96, 300
    x = torch.empty(M, K, dtype=torch.bfloat16, device=DEV)
    x.normal_(generator=torch.Generator(DEV).manual_seed(1))
    a = empty(M, K, 0)
    B.sphinx_q8_quantise(B.BF16, x, K, M, K, False, *a)
    end = x[-last:].contiguous()
    few = empty(last, K, 0)
    B.sphinx_q8_quantise(B.BF16, end, K, last, K, False, *few)
    wide = (K + 127) // 128
    assert torch.equal(a[0][-last * wide * 128:], few[0])
    scales = lambda t: t.view(-1, (wide + 15) // 16 * 16)[:, :wide]  # noqa: E731
    assert torch.equal(scales(a[1])[-last:], scales(few[1]))
    t, tall = empty(K, M, 0), (M + 127) // 128
    B.sphinx_q8_quantise(B.BF16, x, K, M, K, False, None, None, *t)
    del x
    b = pack(numbers(N, K, 3))
    # (not to the bit: beside few rows the contraction is cut)
    c, size = Q.matmul(values(*few, last, K), values(*b, N, K))
    tol = tolerance("bf16", c, size, K)
    assert (np.abs(host(product("bf16", a, b, M, N, K)[-last:]) - c) <= tol).all()
    assert (np.abs(host(product("bf16", b, a, N, M, K)[:, -last:]) - c.T) <= tol.T).all()  # on the other side
    # the transposed copy's last column is the first one's of the columns reversed
    v = t[0].view(K, tall * 128)[-1, :M].view(torch.float8_e4m3fn).float()
    e = torch.exp2(t[1].view(K, -1)[-1, :tall].float() - 127).repeat_interleave(128)[:M]
    r = a[0].view(M, wide * 128)[:, K - 1].view(torch.float8_e4m3fn).float()
    f = torch.exp2(scales(a[1])[:, -1].float() - 127)
    # one number in two groupings: each within half a step (2^-4 of it, or 2^-10 of its unit)
    assert ((v * e - r * f).abs() <= 2.0 ** -3 * (r * f).abs() * 1.1 + 2.0 ** -9 * torch.maximum(e, f)).all()


def test_a_linear_layer_with_its_norm_forward_and_backward():
    """norm -> 8 bits -> product + bias, and back: every gradient against the oracle's, which starts from the values
    that the 8-bit matrices hold."""
    lens, N, K = [100, 0, 57], 200, 136
    M, cu = sum(lens), np.array([0, 100, 100, 157])
    rng = np.random.default_rng(11)
    x, w, b = dev(rng.normal(size=(M, K)) + 0.2), dev(rng.normal(size=(3, K))), dev(rng.normal(size=(3, K)))
    weight, bias = rng.normal(size=(N, K)) / 12, dev(rng.normal(size=N))
    dz = dev(rng.normal(size=(M, N)), "bf16")
    wq, ws = empty(N, K)
    wqt, wst = empty(K, N)
    B.sphinx_q8_quantise(B.F32, dev(weight), K, N, K, True, wq, ws, wqt, wst)
    yq, ys = empty(M, K)
    stats, y = torch.empty(M, 2, device=DEV), torch.empty(M, K, device=DEV)
    norm = (x, K, w, b, K, True, cu)
    B.sphinx_layer_norm_q8(B.F32, B.F32, K, 1e-6, *norm, yq, ys, stats)
    B.sphinx_layer_norm(B.F32, B.F32, B.F32, K, 1e-6, *norm, y, K)
    # the fused form quantises what the other one stores
    assert np.array_equal(values(yq, ys, M, K), Q.quantise(host(y)))
    z = product("bf16", (yq, ys), (wq, ws), M, N, K, bias)
    wv, yv = values(wq, ws, N, K), values(yq, ys, M, K)
    assert np.array_equal(values(wqt, wst, K, N), wv.T)
    c, size = Q.matmul(yv, wv, host(bias))
    assert (np.abs(host(z) - c) <= tolerance("bf16", c, size + np.abs(c), K)).all()
    # backward: dz in both orientations and its sums, the norm's output transposed
    dq, ds = empty(M, N)
    dqt, dst = empty(N, M)
    yqt, yst = empty(K, M)
    db = torch.empty(N, device=DEV)
    wsp = torch.empty(B.sphinx_q8_quantise_workspace_bytes(M, N), dtype=torch.uint8, device=DEV)
    B.sphinx_q8_quantise(B.BF16, dz, N, M, N, False, dq, ds, dqt, dst, db, wsp)
    B.sphinx_q8_quantise(B.F32, y, K, M, K, False, None, None, yqt, yst)
    dy = product("f32", (dq, ds), (wqt, wst), M, K, N)
    dweight = product("f32", (dqt, dst), (yqt, yst), N, K, M)
    c, size = Q.matmul(Q.quantise(host(dz)), wv.T)
    assert (np.abs(host(dy) - c) <= tolerance("f32", c, size, N)).all()
    c, size = Q.matmul(Q.quantise(host(dz).T), Q.quantise(host(y).T))
    assert (np.abs(host(dweight) - c) <= tolerance("f32", c, size, M)).all()
    dx, dw, dshift = torch.empty_like(x), torch.empty(3, K, device=DEV), torch.empty(3, K, device=DEV)
    wsn = torch.empty(B.sphinx_layer_norm_backward_workspace_bytes(K, cu), dtype=torch.uint8, device=DEV)
    B.sphinx_layer_norm_backward(B.F32, B.F32, B.F32, K, x, K, stats, w, K, True, cu, dy.contiguous(), K, dx, K, dw,
                                 dshift, K, wsn)
    want = Q.layer_norm_backward(host(x), host(stats), host(w), cu, True, host(dy))
    # sums of at most 160 numbers of size 10: 200 roundings of 2000 at most
    for got, ref in zip((dx, dw, dshift), want):
        assert np.abs(host(got) - ref).max() <= 200 * U * 2000
