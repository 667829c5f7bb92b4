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


# rows and columns that no tile divides, and contractions that end inside a block and inside a group of four or sixteen
VALUES = [("256x256", 32003, 300, 9), ("256x256", 20001, 520, 18), ("256x256", 6001, 2051, 5), ("192x256", 24001, 300, 10),
          ("192x256", 4001, 2051, 9), ("128x128", 20001, 200, 6), ("128x128", 5003, 777, 11), ("128x64", 16001, 70, 19),
          ("128x64", 16001, 70, 33), ("64x64", 5003, 70, 9)]


@pytest.mark.parametrize("tile, M, N, blocks", VALUES)
def test_values_in_bf16(tile, M, N, blocks):
    check_values(L.BF16, "bf16", tile, M, N, 128 * blocks - 40)


@pytest.mark.parametrize("tile, M, N, blocks", [("192x256", 4001, 2051, 9), ("192x256", 9677, 777, 18),
                                                ("128x128", 20001, 200, 6), ("128x128", 5003, 777, 11),
                                                ("128x64", 16001, 70, 19), ("64x64", 5003, 70, 9)])
def test_values_in_fp32(tile, M, N, blocks):
    check_values(L.F32, "f32", tile, M, N, 128 * blocks - 40)


def check_values(kind, odt, tile, M, N, K):
    for gelu in (False, True):
        assert plan(kind, gelu, M, N, (K + 127) // 128) == (TILES.index(tile), 1)
    a, b, c, size = operands(M, N, K)
    rng = np.random.default_rng(3)
    bias = dev(rng.normal(size=N), "bf16")
    z = c + bias.double()
    lost = sum_error(K, size + z.abs(), odt == "bf16")
    assert within(product(odt, a, b, M, N, K, bias, "bf16", ld=3), z, lost, HALF[odt])
    # GELU has a slope of at most 1.13; its own arithmetic adds 16 roundings of z and its result
    g = 0.5 * z * (1 + torch.tanh(np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3)))
    assert within(product(odt, a, b, M, N, K, bias, "bf16", B.Q8_GELU), g, 1.13 * lost + 16 * U * (z.abs() + 1), HALF[odt])
    before = dev(rng.normal(size=(M, N)), odt)
    total = c + before.double()
    lost = sum_error(K, size + total.abs(), odt == "bf16")
    assert within(product(odt, a, b, M, N, K, epilogue=B.Q8_ADD, before=before, ld=8), total, lost, HALF[odt])


# the QKV product: the first third of the columns is scaled, and ends inside a tile of 256
@pytest.mark.parametrize("tile, M, D", [("few", 7, 1152), ("64x64", 70, 1152), ("128x64", 2501, 384), ("128x128", 2001, 768),
                                        ("192x256", 2501, 1152), ("256x256", 4001, 1152)])
def test_scaled_columns(tile, M, D):
    N, K, scale = 3 * D, D, 0.18
    assert plan(L.BF16, False, M, N, K // 128, True) == (TILES.index(tile), 1)
    a, b, c, size = operands(M, N, K)
    bias = dev(np.random.default_rng(3).normal(size=N), "bf16")
    out = torch.full((M * N + 16,), GUARD, dtype=torch.bfloat16, device=DEV)
    assert L.launch(B.lib(), L.BF16, M, N, K, a, b, bias=bias, bias_bf16=True, out=out, ldo=N, qcols=D, qscale=scale,
                    stream=torch.cuda.current_stream().cuda_stream) == 0
    c = c + bias.double()
    lost = sum_error(K, size + c.abs())
    times = torch.ones(N, dtype=torch.float64, device=DEV)
    times[:D] = float(np.float32(scale))
    # the scaling rounds once more
    assert within(out[:M * N].view(M, N), c * times, (lost + U * (c.abs() + lost)) * times, HALF["bf16"])
    assert (out[M * N:] == GUARD).all()


# the second MLP layer into the residual: out += (1 + gate[row_of]) C
@pytest.mark.parametrize("tile, M, N, blocks", [("64x64", 70, 128, 5), ("128x64", 7001, 516, 9), ("128x128", 2001, 2052, 9),
                                                ("128x128", 8005, 516, 9), ("192x256", 4001, 2052, 9),
                                                ("192x256", 16001, 516, 9), ("192x256", 9677, 1024, 32),
                                                ("256x256", 6001, 2052, 5), ("256x256", 20001, 516, 19)])
def test_gated_residual(tile, M, N, blocks):
    K = 128 * blocks - (0 if blocks == 32 else 40)
    assert plan(L.GATED, False, M, N, blocks) == (TILES.index(tile), 1)
    a, b, c, size = operands(M, N, K)
    rng = np.random.default_rng(3)
    bias = dev(rng.normal(size=N), "bf16")
    c = c + bias.double()
    lost = sum_error(K, size + c.abs())
    G, ldo, ldg = 14, N + 4, N + 8
    gate = dev(rng.normal(size=(G, ldg)))
    cuts = np.sort(np.concatenate([[0, 5, 37, M // 3, min(M, M // 3 + 64)], rng.integers(0, M + 1, G - 5), [M]]))
    runs = np.repeat(np.arange(G), np.diff(cuts))
    # one row of gates, runs of rows that end inside a wave's, and one for each row by itself
    for row_of in (np.full(M, 3), runs, rng.integers(0, G, M)):
        rows = torch.from_numpy(row_of.astype(np.int32)).to(DEV)
        buf = torch.full((M * ldo + 16,), GUARD, device=DEV)
        out = buf[:M * ldo].view(M, ldo)
        h = dev(rng.normal(size=(M, N)) * 3)
        out[:, :N] = h
        assert L.launch(B.lib(), L.GATED, M, N, K, a, b, bias=bias, bias_bf16=True, out=buf, ldo=ldo, gate=gate, ldg=ldg,
                        row_of=rows, stream=torch.cuda.current_stream().cuda_stream) == 0
        g = 1 + gate[rows.long(), :N].double()
        want = h.double() + g * c
        # 1 + gate is rounded, and so is its product with C added to h, at once
        assert within(out[:, :N], want, g.abs() * lost + U * g.abs() * (c.abs() + lost), U)
        assert (out[:, N:] == GUARD).all() and (buf[M * ldo:] == GUARD).all()


# the first MLP layer, which leaves 8 bits
@pytest.mark.parametrize("tile, M, N, blocks", [("128x128", 300, 777, 9), ("192x256", 9677, 777, 9),
                                                ("192x256", 24001, 300, 9), ("256x256", 16001, 777, 5),
                                                ("256x256", 12003, 1030, 9)])
@pytest.mark.parametrize("gelu", [False, True])
def test_outputs_in_8_bits(tile, M, N, blocks, gelu):
    K = 128 * blocks - 40
    assert plan(L.BYTES, gelu, M, N, blocks) == (TILES.index(tile), 1)
    a, b, c, size = operands(M, N, K)
    bias = dev(np.random.default_rng(3).normal(size=N), "bf16")
    q, s = empty(M, N)
    B.sphinx_q8_matmul_q8(M, N, K, *a, *b, B.BF16, bias, B.Q8_GELU if gelu else B.Q8_STORE, q, s)
    nq, ns = B.sphinx_q8_bytes(M, N)
    assert (q[nq:] == 5).all() and (s[ns:] == 5).all()
    wide = (N + 127) // 128
    assert (q[:nq].view(M, -1)[:, N:] == 0).all()
    z = c + bias.double()
    lost = sum_error(K, size + z.abs())
    if gelu:
        lost, z = 1.13 * lost + 16 * U * (z.abs() + 1), 0.5 * z * (1 + torch.tanh(np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3)))
    e, v = s[:ns].view(M, -1)[:, :wide].double() - 127, held(q, s, M, N)
    for j in range(wide):
        cols = slice(128 * j, min(N, 128 * j + 128))
        # the scale's rule, A <= 448 2^e and not 448 2^(e - 1), up to what the largest number may be off by
        top, off = z[:, cols].abs().amax(dim=1), lost[:, cols].amax(dim=1)
        limit = 448 * torch.exp2(e[:, j])
        assert bool(((top - off <= limit) & (top + off > limit / 2)).all())
        # half a step of e4m3: 2^-4 of the number, 2^-10 of the unit for its subnormals
        want, err = z[:, cols], lost[:, cols]
        assert bool(((v[:, cols] - want).abs() <= err + 2.0 ** -4 * (want.abs() + err) + 2.0 ** -10 * torch.exp2(e[:, j:j + 1])).all())


@pytest.mark.parametrize("tile, M, N", [("few", 9, 100), ("64x64", 70, 90), ("128x64", 16001, 70), ("128x128", 20001, 200),
                                        ("192x256", 24001, 300)])
@pytest.mark.parametrize("odt", ["bf16", "f32"])
def test_scales_from_end_to_end(tile, M, N, odt):
    """Blocks whose scales lie between 2^-100 and 2^119, the ends among them, on opposite sides of the product."""
    pairs = [(124, -94), (-94, 124), (40, -10), (90, -60), (-30, 60), (15, 15), (124, -94), (-94, 124), (0, 30), (30, 0), (64, -34)]
    K = 128 * len(pairs) - 40
    if tile == "192x256" and odt == "f32":
        M, N = 9677, 777
    assert plan(L.BF16 if odt == "bf16" else L.F32, False, M, N, len(pairs)) == (TILES.index(tile), 1)
    rng = np.random.default_rng(5)
    xa, xb = (np.clip(rng.normal(size=(n, K)), -7, 7) for n in (M, N))
    for k, (ea, eb) in enumerate(pairs):
        cols = slice(128 * k, 128 * k + 128)
        xa[:, cols] = np.ldexp(xa[:, cols], ea + rng.integers(-1, 1, size=(M, 1)))
        xb[:, cols] = np.ldexp(xb[:, cols], eb + rng.integers(0, 2, size=(N, 1)) * (1 if eb < 0 else -1))
    a, b = pack(xa), pack(xb)
    for s, rows in ((a[1], M), (b[1], N)):
        e = s[:rows * 16].view(rows, 16)[:, :len(pairs)].int() - 127
        assert int(e.min()) <= -98 and int(e.max()) >= 116
    va, vb = held(*a, M, K), held(*b, N, K).T.contiguous()
    c, size = va @ vb, va.abs() @ vb.abs()
    assert within(product(odt, a, b, M, N, K, ld=3), c, sum_error(K, size, odt == "bf16"), HALF[odt])


def test_scaled_columns_of_a_long_contraction():
    """Values that would be cut, where there is a workspace, are not where columns are scaled."""
    M, N, K, scale = 70, 130, 40 * 128 - 3, 0.25
    assert plan(L.BF16, False, M, N, 40)[1] > 1
    a, b, c, size = operands(M, N, K)
    ws = torch.full((B.sphinx_q8_matmul_workspace_bytes(B.BF16, M, N, K),), 255, dtype=torch.uint8, device=DEV)
    out = torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
    assert L.launch(B.lib(), L.BF16, M, N, K, a, b, ws, torch.cuda.current_stream().cuda_stream, out=out, ldo=N,
                    qcols=96, qscale=scale) == 0
    times = torch.ones(N, dtype=torch.float64, device=DEV)
    times[:96] = scale
    assert within(out, c * times, sum_error(K, size) * times, HALF["bf16"]) and (ws == 255).all()


def test_one_step_in_large_tiles_against_the_oracle():
    """One block over all tokens of six requests, whose QKV product takes 256x256, the first MLP layer 192x256 and the second
    128x128.  Nearer to the oracle with 8-bit products than to the one without, by the ratio that test_gpu_q8_refine
    derives for such a step from the shares of numbers that two roundings to 8 bits can disagree on."""
    import oracle as O
    import workloads as W

    cfg = W.ModelCfg(D=1024, heads=16, head_dim=64, mlp=2048, L=1, dtype="bf16")
    wl = W.custom("q8_large_tiles", cfg, [W.Request(1, 40, 100)] * 5 + [W.Request(1, 2, 6)], [1.0] * 6, [0.5] * 6, [2] * 6)
    R = S.from_workload(wl, product_dtype="fp8")
    R.reset()
    n = R.step(0)
    assert n == 5003
    tiles = [TILES[plan(kind, gelu, n, rows, cols // 128, True)[0]]
             for kind, gelu, rows, cols in ((L.BF16, False, 3 * cfg.D, cfg.D), (L.BYTES, True, cfg.mlp, cfg.D),
                                            (L.GATED, False, cfg.D, cfg.mlp))]
    assert tiles == ["256x256", "192x256", "128x128"]
    got = R.state.cpu().numpy().astype(np.float64)
    ref, plain = (O.refine(wl, precision="model", products8=p, steps=1) for p in (True, False))
    a, b = (float(np.sqrt(((got - x) ** 2).mean())) for x in (ref, plain))
    print(f"[q8 large tiles] rms to the 8-bit oracle {a:.3e}, to the other one {b:.3e}", flush=True)
    assert a <= 0.6 * b
    # and no token alone is off: the farthest token's rms, against what 8 bits move tokens by
    off, moved = ((x.reshape(-1) ** 2).reshape(-1, 16).mean(axis=1) ** 0.5 for x in
                  (to_tokens(wl, got - ref), to_tokens(wl, ref - plain)))
    print(f"[q8 large tiles] farthest token {off.max():.3e}, moved {moved.max():.3e}", flush=True)
    assert off.max() <= moved.max()


def to_tokens(wl, state):
    """[token][16] from the NCHW latents of all requests."""
    flat, out, at = np.asarray(state).reshape(-1), [], 0
    for r in wl.requests:
        z = flat[at:at + r.frames * 4 * r.h * r.w].reshape(r.frames, 4, r.h // 2, 2, r.w // 2, 2)
        out.append(z.transpose(0, 2, 4, 1, 3, 5).reshape(-1, 16))
        at += r.frames * 4 * r.h * r.w
    return np.concatenate(out)


@pytest.mark.parametrize("rows, cols, additions", [
    # one tile: 3 of a thread's rows, 2 across a wave's, its eight waves in four pairs
    (100, 300, 3 + 2 + 4), (128, 64, 3 + 2 + 4),
    # beside the tiles: a thread's rows, one in 128, then 8 slices and 16 of those
    (300, 64, 3 + 8 + 16), (2048, 333, 16 + 8 + 16),
    # tiles whose sums are joined: four sums of a sixteenth of them, 2 for the four, 16 slices
    (3000, 96, 9 + 2 + 2 + 16), (9677, 40, 9 + 5 + 2 + 16)])
@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_column_sums_are_off_by_their_additions_at_most(rows, cols, additions, name):
    x = dev(numbers(rows, cols), name)
    sums = torch.full((cols + 3,), GUARD, device=DEV)
    ws = torch.full((B.sphinx_q8_quantise_workspace_bytes(rows, cols),), 255, dtype=torch.uint8, device=DEV)
    B.sphinx_q8_quantise(TYPE[name][1], x, cols, rows, cols, False, None, None, None, None, sums, ws)
    err = (sums[:cols].double() - x.double().sum(dim=0)).abs()
    assert bool((err <= 1.01 * additions * U * x.double().abs().sum(dim=0)).all()) and (sums[cols:] == GUARD).all()
