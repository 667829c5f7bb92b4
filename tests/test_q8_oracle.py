"""The oracle of the layer norm and the 8-bit products against itself (differences, hand-made cases), and what the C
entry points and the binding refuse, without a GPU."""
import os

import numpy as np
import pytest

from oracle import q8 as Q

torch = pytest.importorskip("torch")
S = pytest.importorskip("paper_2511_18672_amd")
B = S.binding

if not os.path.exists(B.LIB_PATH):
    pytest.skip("libsphinx.so not built", allow_module_level=True)


# ---- the oracle ------------------------------------------------------------
def test_layer_norm_gradients_against_differences():
    rng = np.random.default_rng(1)
    cu = [0, 3, 3, 7]
    x, w, b, dy = rng.normal(size=(7, 11)), rng.normal(size=(3, 11)), rng.normal(size=(3, 11)), rng.normal(size=(7, 11))
    for plus_one in (False, True):
        loss = lambda x, w, b: float((Q.layer_norm(x, w, b, cu, plus_one, 1e-6)[0] * dy).sum())  # noqa: E731
        dx, dw, db = Q.layer_norm_backward(x, Q.layer_norm(x, w, b, cu, plus_one, 1e-6)[1], w, cu, plus_one, dy)
        for k, (t, grad) in enumerate(((x, dx), (w, dw), (b, db))):
            for at in np.ndindex(t.shape):
                h = 1e-5
                args = [[x, w, b], [x, w, b]]
                for s in (0, 1):
                    moved = t.copy()
                    moved[at] += h if s == 0 else -h
                    args[s][k] = moved
                # a central difference is off by h^2 times the third derivative and 1e-16/h of the loss (about 10)
                assert abs((loss(*args[0]) - loss(*args[1])) / (2 * h) - grad[at]) < 1e-7


def test_layer_norm_gradient_against_autograd():
    rng = np.random.default_rng(2)
    x, w, b, dy = (torch.from_numpy(rng.normal(size=s)).requires_grad_(k < 3)
                   for k, s in enumerate([(9, 40), (40,), (40,), (9, 40)]))
    y = torch.nn.functional.layer_norm(x, (40,), w, b, 1e-5)
    y.backward(dy)
    ref, stats = Q.layer_norm(x.detach().numpy(), w.detach().numpy()[None], b.detach().numpy()[None], [0, 9], False, 1e-5)
    dx, dw, db = Q.layer_norm_backward(x.detach().numpy(), stats, w.detach().numpy()[None], [0, 9], False, dy.numpy())
    for got, want in ((ref, y), (dx, x.grad), (dw[0], w.grad), (db[0], b.grad)):
        assert np.allclose(got, want.detach().numpy(), rtol=1e-11, atol=1e-12)


def test_quantised_values():
    x = np.zeros((2, 130))
    x[0, 0], x[0, 1], x[0, 129], x[1, 0] = 448.0, 0.4, -448.5, np.inf
    v = Q.quantise(x)
    assert v[0, 0] == 448.0 and v[0, 1] == 0.40625 and v[0, 129] == -448.0 and np.isnan(v[1, 0]) and v[1, 1] == 0.0
    e = Q.exponents(x)
    assert e[0, 0] == 0 and e[0, 129] == 1 and e[1, 0] == -100
    assert (Q.exponents(x, True)[:, 0] == 0).all() and (Q.exponents(x, True)[:, 129] == 1).all()
    assert np.array_equal(Q.quantise(x[:1], True), Q.quantise(x[:1].T, True).T)
    big = np.full((1, 2), 2.0 ** 127.9)
    assert Q.exponents(big)[0, 0] == 119 and Q.quantise(big)[0, 0] == 448.0 * 2.0 ** 119


# ---- refusals of the C entry points -----------------------------------------
def status(fn, *args):
    return getattr(B.lib(), fn)(*args)


OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
P = 1 << 20  # a pointer that no refused call looks at


def cu(*v):
    return np.array(v, np.int32).tobytes()


def norm(xdt=1, wdt=0, ydt=1, cols=64, eps=1e-6, x=P, ldx=64, w=P, b=P, ldw=64, one=1, bounds=(0, 4), y=P, ldy=64,
         stats=P):
    return status("sphinx_layer_norm", xdt, wdt, ydt, cols, eps, x, ldx, w, b, ldw, one, cu(*bounds), len(bounds) - 1,
                  y, ldy, stats, None)


@pytest.mark.parametrize("bad, want", [
    (dict(xdt=2), UNSUPPORTED), (dict(wdt=-1), UNSUPPORTED), (dict(ydt=7), UNSUPPORTED), (dict(cols=0), INVALID),
    (dict(cols=16385, ldx=20000, ldw=20000, ldy=20000), UNSUPPORTED), (dict(eps=-1.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(x=None), INVALID), (dict(x=P + 8), INVALID), (dict(ldx=63), INVALID),
    (dict(ldw=63), INVALID), (dict(one=2), INVALID), (dict(bounds=(0,)), INVALID), (dict(bounds=(1, 4)), INVALID),
    (dict(bounds=(0, 4, 3)), INVALID), (dict(bounds=(0, (1 << 30) + 1)), UNSUPPORTED), (dict(bounds=tuple(range(66))), UNSUPPORTED), (dict(y=None), INVALID),
    (dict(y=P + 4), INVALID), (dict(ldy=1), INVALID), (dict(stats=P + 8), INVALID), (dict(w=P + 2), INVALID),
])
def test_norm_refuses(bad, want):
    assert norm(**bad) == want


def test_norm_of_no_rows_is_a_no_op():
    assert norm(bounds=(0, 0, 0), x=None, y=None, stats=None) == OK
    assert status("sphinx_layer_norm_q8", 0, 0, 64, 1e-6, None, 64, None, None, 0, 0, cu(0, 0), 1, None, None, None,
                  None) == OK
    assert status("sphinx_layer_norm_q8", 0, 0, 64, 1e-6, P, 64, None, None, 0, 0, cu(0, 1), 1, None, P, None,
                  None) == INVALID


def backward(xdt=1, wdt=0, gdt=1, cols=64, x=P, ldx=64, stats=P, w=P, ldw=64, one=0, bounds=(0, 4), dy=P, lddy=64,
             dx=P, lddx=64, dw=P, db=P, ldg=64, ws=P, ws_bytes=1 << 20):
    return status("sphinx_layer_norm_backward", xdt, wdt, gdt, cols, x, ldx, stats, w, ldw, one, cu(*bounds),
                  len(bounds) - 1, dy, lddy, dx, lddx, dw, db, ldg, ws, ws_bytes, None)


@pytest.mark.parametrize("bad, want", [
    (dict(xdt=3), UNSUPPORTED), (dict(gdt=3), UNSUPPORTED), (dict(cols=0), INVALID), (dict(stats=None), INVALID),
    (dict(dy=None), INVALID), (dict(lddy=63), INVALID), (dict(lddx=63), INVALID), (dict(ldg=63), INVALID),
    (dict(ws=None), INVALID), (dict(ws=P + 128), INVALID), (dict(ws_bytes=16), WORKSPACE), (dict(dx=P + 2), INVALID),
    (dict(dw=P + 8), INVALID), (dict(bounds=(0, 5, 4)), INVALID),
])
def test_norm_backward_refuses(bad, want):
    assert backward(**bad) == want


def test_norm_backward_without_outputs_or_rows():
    assert backward(dx=None, dw=None, db=None, ws=None, ws_bytes=0) == OK
    assert backward(bounds=(0, 0), x=None, stats=None, dy=None, dw=None, db=None, ws=None, ws_bytes=0) == OK


def quant(dt=1, x=P, ldx=200, rows=100, cols=200, square=0, q=P, s=P, qt=P, st=P, sums=P, ws=P, ws_bytes=1 << 20):
    return status("sphinx_q8_quantise", dt, x, ldx, rows, cols, square, q, s, qt, st, sums, ws, ws_bytes, None)


@pytest.mark.parametrize("bad, want", [
    (dict(dt=2), UNSUPPORTED), (dict(x=None), INVALID), (dict(x=P + 4), INVALID), (dict(ldx=199), INVALID),
    (dict(rows=-1), INVALID), (dict(cols=-1, ldx=0), INVALID), (dict(square=2), INVALID), (dict(s=None), INVALID),
    (dict(st=None), INVALID), (dict(q=None, qt=None, sums=None), INVALID), (dict(q=P + 8), INVALID),
    (dict(ws=None), INVALID), (dict(ws_bytes=799), WORKSPACE), (dict(ws=P + 16), INVALID),
    (dict(cols=(1 << 23) + 1, ldx=1 << 24), UNSUPPORTED), (dict(rows=1 << 28, cols=1 << 10, ldx=1 << 10), UNSUPPORTED), (dict(rows=(1 << 28) + 1), UNSUPPORTED),
    (dict(rows=(1 << 23) + 1), UNSUPPORTED),
])
def test_quantise_refuses(bad, want):
    assert quant(**bad) == want


def test_quantise_of_nothing_is_a_no_op():
    assert quant(rows=0, x=None, sums=None, q=None, s=None, qt=None, st=None) == OK
    assert quant(cols=0, x=None, q=None, s=None, qt=None, st=None, sums=None, ws=None) == OK


def product(odt=1, M=5, N=6, K=7, a=P, sa=P, b=P, sb=P, bdt=0, bias=P, epi=0, out=P, ldo=6, ws=P, ws_bytes=1 << 30):
    return status("sphinx_q8_matmul", odt, M, N, K, a, sa, b, sb, bdt, bias, epi, out, ldo, ws, ws_bytes, None)


@pytest.mark.parametrize("bad, want", [
    (dict(odt=2), UNSUPPORTED), (dict(bdt=2), UNSUPPORTED), (dict(M=-1), INVALID), (dict(K=-1), INVALID),
    (dict(K=(1 << 23) + 1), UNSUPPORTED), (dict(a=None), INVALID), (dict(sb=None), INVALID), (dict(a=P + 8), INVALID),
    (dict(epi=3), INVALID), (dict(epi=-1), INVALID), (dict(out=None), INVALID), (dict(ldo=5), INVALID),
    (dict(out=P + 8), INVALID), (dict(bias=P + 4), INVALID), (dict(ws=P + 64), INVALID),
    (dict(M=1 << 28, N=1 << 23, ldo=1 << 23), UNSUPPORTED), (dict(M=(1 << 28) + 1), UNSUPPORTED),
])
def test_matmul_refuses(bad, want):
    assert product(**bad) == want


def product8(M=5, N=6, K=7, a=P, sa=P, b=P, sb=P, bdt=0, bias=P, epi=0, q=P, s=P):
    return status("sphinx_q8_matmul_q8", M, N, K, a, sa, b, sb, bdt, bias, epi, q, s, None)


@pytest.mark.parametrize("bad, want", [
    (dict(bdt=2), UNSUPPORTED), (dict(N=-1), INVALID), (dict(a=None), INVALID), (dict(sb=P + 8), INVALID),
    (dict(epi=2), INVALID), (dict(q=None), INVALID), (dict(s=None), INVALID), (dict(q=P + 4), INVALID),
    (dict(bias=P + 2), INVALID), (dict(N=(1 << 23) + 1), UNSUPPORTED), (dict(K=(1 << 23) + 1), UNSUPPORTED),
])
def test_matmul_into_8_bits_refuses(bad, want):
    assert product8(**bad) == want


def test_the_8_bit_step_refuses():
    import workloads as W

    reqs = B.make_requests([W.Request(1, 4, 4)])
    good = W.ModelCfg(D=128, heads=2, head_dim=64, mlp=256, L=2, dtype="bf16")
    f32 = W.ModelCfg(D=128, heads=2, head_dim=64, mlp=256, L=2, dtype="f32")
    with pytest.raises(S.SphinxError):
        B.sphinx_model_q8_bytes(B.model_desc(f32, P))
    with pytest.raises(S.SphinxError):
        B.sphinx_refine_q8_workspace_bytes(B.model_desc(f32, P), reqs, 4)
    desc = B.model_desc(good, P)
    # a block: QKV, MLP1 and MLP2, each with a row of 16 scale bytes per row
    assert B.sphinx_model_q8_bytes(desc) == 2 * ((384 * 128 + 384 * 16) + (256 * 128 + 256 * 16) + (128 * 256 + 128 * 16))
    plain, more = B.sphinx_refine_workspace_bytes(desc, reqs, 4), B.sphinx_refine_q8_workspace_bytes(desc, reqs, 4)
    assert more >= plain + 4 * 128 + 4 * 16
    bounds = np.array([0, 4], np.int32)

    def step(w8=P, w8_bytes=1 << 30, cache=None, kv8=0, ws_bytes=1 << 30, d=desc):
        import ctypes

        return status("sphinx_refine_step_q8", ctypes.byref(d), w8, w8_bytes, reqs, 1, P, 4, bounds.ctypes.data, P, P, P,
                      P, cache, kv8, P, ws_bytes, None)

    assert step(w8=None) == INVALID and step(w8=P + 16) == INVALID and step(w8_bytes=100) == WORKSPACE
    assert step(kv8=1) == INVALID and step(kv8=2) == INVALID and step(ws_bytes=plain) == WORKSPACE
    assert step(d=B.model_desc(f32, P)) == UNSUPPORTED


def test_matmul_of_nothing_is_a_no_op():
    assert product(M=0, a=None, sa=None, out=None) == OK
    assert product(N=0, b=None, sb=None, out=None, ldo=0) == OK


def test_sizes():
    assert B.sphinx_q8_bytes(3, 129) == (3 * 256, 3 * 16)
    assert B.sphinx_q8_bytes(2, 17 * 128 + 1) == (2 * 18 * 128, 2 * 32)
    assert B.sphinx_q8_bytes(0, 5) == (0, 0) and B.sphinx_q8_bytes(5, 0) == (0, 0)
    for bad in ((-1, 1), (1, -1), (1, (1 << 23) + 1), ((1 << 28) + 1, 1)):
        with pytest.raises(S.SphinxError):
            B.sphinx_q8_bytes(*bad)
    with pytest.raises(ValueError, match="32 bits"):
        B.sphinx_q8_bytes(1 << 32, 1)
    with pytest.raises(S.SphinxError):
        B.sphinx_layer_norm_backward_workspace_bytes(64, [0, 4, 2])


# ---- refusals of the binding -------------------------------------------------
def zeros(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype)


def test_binding_refuses_tensors_of_another_type_or_too_few():
    x, w, y = zeros(4, 64), zeros(2, 64, dtype=torch.float32), zeros(4, 64)
    call = lambda x=x, w=w, y=y, stats=None, cu=(0, 1, 4): B.sphinx_layer_norm(  # noqa: E731
        B.BF16, B.F32, B.BF16, 64, 1e-6, x, 64, w, w, 64, True, cu, y, 64, stats)
    for bad in (dict(x=x.float()), dict(x=zeros(3, 64)), dict(w=w.bfloat16()), dict(w=zeros(1, 64, dtype=torch.float32)), dict(y=zeros(4, 32)),
                dict(y=zeros(1, 64).expand(4, 64)), dict(stats=zeros(8)), dict(stats=zeros(7, dtype=torch.float32)),
                dict(cu=[0]), dict(cu=[0.0, 4.0])):
        with pytest.raises(ValueError):
            call(**bad)
    u8 = lambda n: torch.zeros(n, dtype=torch.uint8)  # noqa: E731
    for q, s in ((u8(511), u8(64)), (u8(512), u8(63)), (u8(512), None), (zeros(512), u8(64)), (u8(1024)[::2], u8(64))):
        with pytest.raises(ValueError):
            B.sphinx_q8_quantise(B.BF16, x, 64, 4, 64, False, q, s)
        with pytest.raises(ValueError):
            B.sphinx_layer_norm_q8(B.BF16, B.F32, 64, 1e-6, x, 64, None, None, 64, False, [0, 4], q, s)
        with pytest.raises(ValueError):
            B.sphinx_q8_matmul(B.BF16, 4, 4, 64, q, s, u8(512), u8(64), B.F32, None, B.Q8_STORE, zeros(4, 4), 4, None)
    with pytest.raises(ValueError, match="bias"):
        B.sphinx_q8_matmul(B.BF16, 4, 4, 64, u8(512), u8(64), u8(512), u8(64), B.F32, zeros(4), B.Q8_STORE,
                           zeros(4, 4), 4, None)
    with pytest.raises(ValueError, match="out"):
        B.sphinx_q8_matmul(B.BF16, 4, 4, 64, u8(512), u8(64), u8(512), u8(64), B.F32, None, B.Q8_STORE, zeros(3, 4), 4,
                           None)
    f = torch.float32
    with pytest.raises(ValueError, match="dw"):
        B.sphinx_layer_norm_backward(B.BF16, B.F32, B.BF16, 64, x, 64, zeros(8, dtype=f), w, 64, True, [0, 1, 4], x, 64, x,
                                     64, zeros(2, 64), None, 64, None)
    with pytest.raises(ValueError, match="stats"):
        B.sphinx_layer_norm_backward(B.BF16, B.F32, B.BF16, 64, x, 64, zeros(7, dtype=f), w, 64, True, [0, 1, 4], x, 64, x,
                                     64, None, None, 64, None)
