"""Products that leave a matrix in 8 bits, and the refinement step with its QKV and MLP products in 8 bits."""
import dataclasses

import numpy as np
import pytest

import oracle as O
import workloads as W
from oracle import q8 as Q

torch = pytest.importorskip("torch")
S = pytest.importorskip("paper_2511_18672_amd")
B = S.binding

from test_gpu_q8 import SHAPES, U, dev, empty, host, numbers, pack, product, values  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M, N, K", SHAPES + [(2000, 1100, 300), (9000, 2048, 256)])
@pytest.mark.parametrize("gelu", [False, True])
def test_product_in_8_bits(M, N, K, gelu):
    a, b = pack(numbers(M, K, 1)), pack(numbers(N, K, 2) / np.sqrt(K))
    bias = dev(np.random.default_rng(3).normal(size=N), "bf16")
    q, s = empty(M, N)
    B.sphinx_q8_matmul_q8(M, N, K, *a, *b, B.BF16, bias, B.Q8_GELU if gelu else B.Q8_STORE, q, s)
    nq, ns = B.sphinx_q8_bytes(M, N)
    assert (q[nq:] == 5).all() and (s[ns:] == 5).all()
    c, size = Q.matmul(values(*a, M, K), values(*b, N, K), host(bias))
    want = Q.gelu(c) if gelu else c
    size = size + np.abs(c)
    # as for bf16 outputs before their rounding; GELU has a slope of at most 1.13 and 16 roundings of its own
    tol = ((K / 4 + 8) * U + 2.0 ** -10) * size * (1.13 if gelu else 1.0) + 16 * U * (np.abs(c) + 1)
    got = values(q, s, M, N)
    wide = (N + 127) // 128
    e = s[:ns].view(M, -1)[:, :wide].cpu().numpy().astype(np.int64) - 127
    e, ref = np.repeat(e, 128, axis=1)[:, :N], Q.exponents(want)
    near = np.zeros_like(want, bool)  # groups whose largest number is within its error of a border between scales
    for j in range(0, N, 128):
        top, lost = np.abs(want[:, j:j + 128]).max(axis=1), tol[:, j:j + 128].max(axis=1)
        border = 448.0 * np.ldexp(1.0, ref[:, j])
        near[:, j:j + 128] = (np.minimum(np.abs(top - border), np.abs(top - border / 2)) <= lost)[:, None]
    assert ((e == ref) | near).all()
    assert (np.abs(got - want) <= tol + 2.0 ** -4 * (np.abs(want) + tol) + np.ldexp(2.0 ** -10, e)).all()


def test_product_in_8_bits_is_the_other_one_quantised():
    """Both start from the same fp32 sums: the bf16 outputs are the same numbers rounded to 8 bits, so the two differ by
    an 8-bit and a bf16 half step."""
    M, N, K = 300, 384, 700
    a, b = pack(numbers(M, K, 1)), pack(numbers(N, K, 2))
    q, s = empty(M, N)
    B.sphinx_q8_matmul_q8(M, N, K, *a, *b, B.F32, None, B.Q8_STORE, q, s)
    wide = host(product("bf16", a, b, M, N, K))
    e = np.repeat(s[:M * 16].view(M, 16)[:, :3].cpu().numpy().astype(np.int64) - 127, 128, axis=1)
    assert (np.abs(values(q, s, M, N) - wide) <= (2.0 ** -4 + 2.0 ** -8) * 1.01 * np.abs(wide) + np.ldexp(2.0 ** -10, e)).all()


def test_product_in_8_bits_of_what_is_not_finite():
    xa, xb = numbers(150, 300, 7), numbers(260, 300, 8)
    ref = [t.clone() for t in empty(150, 260)]
    B.sphinx_q8_matmul_q8(150, 260, 300, *pack(xa), *pack(xb), B.F32, None, B.Q8_STORE, *ref)
    xa[3, 0], xb[200, 5] = np.nan, np.nan
    q, s = empty(150, 260)
    B.sphinx_q8_matmul_q8(150, 260, 300, *pack(xa), *pack(xb), B.F32, None, B.Q8_STORE, q, s)
    got, want = values(q, s, 150, 260), values(*ref, 150, 260)
    assert np.isnan(got[3]).all() and np.isnan(got[:, 200]).all()
    rows = np.arange(150) != 3
    cols = (np.arange(260) < 128) | (np.arange(260) >= 256)  # the NaN column's block may take another scale
    assert np.array_equal(got[np.ix_(rows, cols)], want[np.ix_(rows, cols)])
    assert np.isfinite(got[np.ix_(rows, np.arange(260) != 200)]).all()


MODELS = {"64": W.ModelCfg(D=256, heads=4, head_dim=64, mlp=1024, L=3, dtype="bf16"),
          "72": W.ModelCfg(D=1152, heads=16, head_dim=72, mlp=384, L=2, dtype="bf16")}


def workload(model, attention="joint"):
    shapes = [W.Request(3, 24, 20), W.Request(2, 10, 14), W.Request(1, 4, 4)]
    cfg = dataclasses.replace(MODELS[model], attention=attention)
    return W.custom(f"q8_steps_{model}_{attention}", cfg, shapes, [0.4, 0.7, 0.5], [("uniform", 0.3, 0.7), 0.5, 0.2],
                    [4, 3, 3])


@pytest.mark.parametrize("model", list(MODELS))
def test_weights_are_quantised_in_squares(model):
    wl = workload(model)
    R = S.from_workload(wl, product_dtype="fp8")
    w8, at, cfg = R.w8.cpu(), 0, wl.model
    for l in range(cfg.L):
        for name in ("qkv_w", "fc1_w", "fc2_w"):
            w = np.asarray(wl.weights[f"b{l}.{name}"], np.float64)
            nq, ns = B.sphinx_q8_bytes(*w.shape)
            q = w8[at:at + nq]
            at += (nq + 255) // 256 * 256
            s = w8[at:at + ns]
            at += (ns + 255) // 256 * 256
            assert np.array_equal(values(q, s, *w.shape), Q.quantise(w, square=True))
    assert at == w8.numel()


@pytest.mark.parametrize("model, kw", [("64", {}), ("72", {}), ("64", dict(attention="factorised")),
                                       ("64", dict(cache_period=2)), ("72", dict(cache_period=2, cache_dtype="fp8")),
                                       ("64", dict(attention="factorised", cache_period=2, cache_dtype="fp8"))])
def test_loop_against_the_oracle(model, kw):
    """The latents are nearer to the oracle with 8-bit products than to the one without.  There is no bound on the
    largest difference: where two roundings to 8 bits start from numbers that differ in bf16, one in tens falls to the
    other side, by a whole step (2^-3 of it), and the next block starts from that."""
    kw = dict(kw)
    wl = workload(model, kw.pop("attention", "joint"))
    got = S.from_workload(wl, product_dtype="fp8", **kw).run().cpu().numpy().astype(np.float64)
    okw = dict(period=kw.get("cache_period", 0), cache8=kw.get("cache_dtype") == "fp8")
    ref, plain = (O.refine(wl, precision="model", products8=p, **okw) for p in (True, False))
    a, b = (float(np.sqrt(((got - x) ** 2).mean())) for x in (ref, plain))
    print(f"[q8 loop {model} {kw}] rms to the 8-bit oracle {a:.3e}, to the other one {b:.3e}", flush=True)
    assert a < b


@pytest.mark.parametrize("model", list(MODELS))
def test_one_step_of_one_block_against_the_oracle(model):
    """A number x is quantised in steps of D = 2^-3.5 |x| (between 2^-4 and 2^-3), which is an error of variance D^2/12.
    The GPU's number and the oracle's differ by some d, and fall to different sides of a border with probability d/D: an
    error of variance d D, 12 d/D of the other.  The first norm's input is fp32 throughout: d/D below 10^-4.  The second
    norm's comes through an attention in bf16 (o is rounded: d = 2^-8 of its part of the residual stream at most) and
    the GELU's through it and a product: even if that were all of them, 12 d/D = 12 2^-8 2^3.5 = 0.53, of the roundings
    of two of the three inputs.  The ratio of the rms is then below sqrt(0.53 2/3) < 0.6."""
    wl = workload(model)
    wl = dataclasses.replace(wl, model=dataclasses.replace(wl.model, L=1))
    R = S.from_workload(wl, product_dtype="fp8")
    R.reset()
    R.step(0)
    got = R.state.cpu().numpy().astype(np.float64)
    ref, plain = (O.refine(wl, precision="model", products8=p, steps=1) for p in (True, False))
    a, b = (float(np.sqrt(((got - x) ** 2).mean())) for x in (ref, plain))
    print(f"[q8 step {model}] rms to the 8-bit oracle {a:.3e}, to the other one {b:.3e}", flush=True)
    assert a <= 0.6 * b


def test_the_loop_repeats_bit_for_bit():
    wl = workload("64")
    one, two = (S.from_workload(wl, product_dtype="fp8").run().cpu() for _ in range(2))
    assert torch.equal(one, two)


def test_refusals():
    wl = workload("64")
    with pytest.raises(ValueError, match="product_dtype"):
        S.from_workload(wl, product_dtype="int4")
    f32 = W.custom("f32", W.ModelCfg(D=64, heads=1, head_dim=64, mlp=128, L=1, dtype="f32"), [W.Request(1, 4, 4)], [0.5],
                   [0.5], [2])
    with pytest.raises(ValueError, match="bf16"):
        S.from_workload(f32, product_dtype="fp8")
