"""The 8-bit cache's oracle against properties of its definition, and the calls'
refusals through the C ABI (no GPU needed)."""
import ctypes
import os

import numpy as np
import pytest

import oracle as O
import workloads as W

S = pytest.importorskip("paper_2511_18672_amd")
torch = pytest.importorskip("torch")

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(S.binding.LIB_PATH):
        pytest.skip("libsphinx.so not built")
    return S.lib()


def test_e4m3_numbers_are_the_type():
    codes = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(O.kv8.e4m3_numbers(), codes)


def test_rounding_is_nearest_even():
    x = np.random.default_rng(0).standard_normal(4000) * 2.0 ** np.random.default_rng(1).integers(-12, 8, 4000)
    x = np.concatenate([x, O.kv8.e4m3_numbers(), (O.kv8.e4m3_numbers()[1:] + O.kv8.e4m3_numbers()[:-1]) / 2])
    x = np.clip(x, -448, 448).astype(np.float32)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(O.kv8.round_e4m3(x), want)
    y = O.kv8.round_e4m3(np.array([np.inf, -np.inf, np.nan, 460.0, -1e9]))
    assert np.isnan(y[:3]).all() and list(y[3:]) == [448.0, -448.0]


@pytest.mark.parametrize("top,e", [(448.0, 0), (449.0, 1), (224.0, -1), (1.0, -8), (0.0, -100), (1e-44, -100),
                                   (3.4e38, 119), (1.75, -8), (1.7500001, -7)])
def test_block_exponent(top, e):
    assert O.kv8.block_exponent(np.array([0.0, -top, np.inf, np.nan])) == e


def test_quantise_error_and_idempotence():
    rng = np.random.default_rng(2)
    bounds = [0, 1, 65, 65, 200]
    x = rng.standard_normal((200, 3, 64)) * np.exp(rng.standard_normal((200, 1, 1)))
    q = O.kv8.quantise(x, bounds)
    assert np.array_equal(O.kv8.quantise(q, bounds), q)
    for a, b in O.kv8.blocks(bounds):
        for h in range(3):
            step = 2.0 ** (O.kv8.block_exponent(x[a:b, h]) - 9)
            # half a step: 2^-4 of the value, or half the smallest step
            assert (np.abs(q[a:b, h] - x[a:b, h]) <= np.maximum(np.abs(x[a:b, h]) * 2.0 ** -4, step / 2)).all()


def test_write_keeps_other_rows():
    rng = np.random.default_rng(3)
    bounds = [0, 130]
    held = O.kv8.quantise(rng.standard_normal((130, 2, 64)), bounds)
    got = O.kv8.write(held, rng.standard_normal((3, 2, 64)) * 0.5, np.array([5, 6, -1]), bounds)
    keep = np.ones(130, bool)
    keep[[5, 6]] = False
    assert np.array_equal(got[keep], held[keep])  # the scale did not grow
    assert not np.array_equal(got[~keep], held[~keep])


def test_oracle_attention_shares_heads_and_allows_no_keys():
    rng = np.random.default_rng(4)
    q, k, v = rng.standard_normal((3, 4, 8)), rng.standard_normal((5, 2, 8)), rng.standard_normal((5, 2, 8))
    o, _, _ = O.kv8.attention(q, k, v, [0, 2, 3], [0, 5, 5])
    assert (o[2] == 0).all()
    s = np.exp2(q[1, 3] @ k[:, 1].T)
    assert np.allclose(o[1, 3], s @ v[:, 1] / s.sum())
    assert np.allclose(O.attention(q[:2].reshape(2, 32) * 0 + 1, np.repeat(k, 2, 1).reshape(5, 32),
                                   np.repeat(v, 2, 1).reshape(5, 32), 4, np.array([0, 2]), kv_seg=np.array([0, 5]),
                                   scale=np.log(2.0)),
                       O.kv8.attention(np.ones((2, 4, 8)), k, v, [0, 2], [0, 5])[0].reshape(2, 32))


def _cu(*v):
    return (ctypes.c_int32 * len(v))(*v)


def test_bytes_and_their_refusals(L):
    out = ctypes.c_size_t()
    f = lambda hk, d, cu, n: L.sphinx_kv8_bytes(hk, d, cu, n, ctypes.byref(out))
    # 3 blocks (1 + 0 + 2) of 2 heads: keys and values of 64 rows, and two scale bytes a block and head
    assert f(2, 64, _cu(0, 1, 1, 66), 3) == OK and out.value == 3 * 2 * 2 * 64 * 64 + 256
    assert f(1, 72, _cu(0, 64), 1) == OK and out.value == 2 * 64 * 72 + 256
    assert f(1, 64, _cu(0, 0), 1) == OK and out.value == 0
    assert f(1, 32, _cu(0, 64), 1) == UNSUPPORTED
    assert f(0, 64, _cu(0, 64), 1) == INVALID
    assert f(1, 64, _cu(1, 64), 1) == INVALID
    assert f(1, 64, _cu(0, 64, 63), 2) == INVALID
    assert f(1, 64, None, 1) == INVALID
    assert f(1, 64, _cu(0, 64), 0) == INVALID
    assert f(1, 64, _cu(*range(66)), 65) == UNSUPPORTED
    assert f(2048, 64, _cu(0, 64), 1) == UNSUPPORTED
    assert f(32, 64, _cu(0, (1 << 31) - 1), 1) == UNSUPPORTED  # 2^31 tiles
    assert L.sphinx_kv8_bytes(1, 64, _cu(0, 64), 1, None) == INVALID
    # long caches: sizes past 32 bits
    assert f(16, 64, _cu(0, 1 << 30), 1) == OK and out.value == (1 << 30) * 2048 + (1 << 24) * 16 * 2


@pytest.mark.parametrize("load", [False, True])
def test_store_and_load_refusals(L, load):
    P = ctypes.c_void_p

    def call(dt=1, hk=1, d=64, k=256, v=256, ld=64, idx=256, n=3, cu=_cu(0, 8), nseg=1, c=256, have=1 << 40):
        if load:
            return L.sphinx_kv8_load(dt, hk, d, P(c), have, cu, nseg, P(idx), n, P(k), P(v), ld, None)
        return L.sphinx_kv8_store(dt, hk, d, P(k), P(v), ld, P(idx), n, cu, nseg, P(c), have, None)

    assert call(dt=2) == UNSUPPORTED
    assert call(d=80, ld=80) == UNSUPPORTED
    assert call(ld=56) == INVALID and call(ld=68) == INVALID and call(hk=2) == INVALID
    assert call(n=-1) == INVALID
    assert call(hk=2, ld=128, n=1 << 29) == UNSUPPORTED  # 2^31 rows of all tiles
    assert call(idx=None, n=9) == INVALID  # more rows than tokens
    for kw in (dict(k=None), dict(v=None), dict(c=None), dict(k=264), dict(v=8), dict(c=260), dict(idx=4)):
        assert call(**kw) == INVALID, kw
    assert call(cu=_cu(0, 8, 4), nseg=2) == INVALID
    assert call(have=2 * 64 * 64 + 255) == WORKSPACE  # a block of one head needs 256 more than its tiles
    assert call(n=0, k=None, v=None, c=None, idx=None) == OK  # nothing to do
    assert call(cu=_cu(0, 0), n=5, k=None, v=None, c=None) == OK  # no tokens: every row is skipped


@pytest.mark.parametrize("call", ["store", "load"])
def test_index_tensors_that_are_not_int32_in_a_row_are_refused(call):
    torch = pytest.importorskip("torch")
    from paper_2511_18672_amd import binding as B
    rows, cache = torch.zeros(8, 64), torch.zeros(8192, dtype=torch.uint8)
    good = torch.arange(8, dtype=torch.int32)
    for idx in (good.long(), good.float(), good[:7], torch.arange(16, dtype=torch.int32)[::2]):
        with pytest.raises(ValueError, match="int32"):
            if call == "store":
                B.sphinx_kv8_store(B.F32, 1, 64, rows, rows, 64, idx, 8, [0, 64], cache)
            else:
                B.sphinx_kv8_load(B.F32, 1, 64, cache, [0, 64], idx, 8, rows, rows, 64)


def test_attention_refusals(L):
    P = ctypes.c_void_p
    need = ctypes.c_size_t()

    def size(dt=1, h=2, hk=1, d=64, cq=_cu(0, 4), ck=_cu(0, 8), nseg=1, out=need):
        return L.sphinx_kv8_attention_workspace_bytes(dt, h, hk, d, cq, ck, nseg, None if out is None else ctypes.byref(out))

    def call(dt=1, h=2, hk=1, d=64, q=256, ldq=128, c=256, cq=_cu(0, 4), ck=_cu(0, 8), kl=None, nseg=1, o=256, ws=256,
             nbytes=1 << 40, have=1 << 40):
        return L.sphinx_kv8_attention(dt, h, hk, d, P(q), ldq, P(c), have, cq, ck, kl, nseg, P(o), P(ws), nbytes,
                                      None)

    assert size() == OK and need.value > 0
    for f in (size, call):
        assert f(dt=7) == UNSUPPORTED
        assert f(dt=0, d=72, **({} if f is size else dict(ldq=144))) == UNSUPPORTED  # fp32: head_dim 64
        assert f(d=128) == UNSUPPORTED
        assert f(h=3, hk=2) == INVALID and f(h=0) == INVALID and f(hk=0) == INVALID
        assert f(cq=None) == INVALID and f(ck=None) == INVALID
        assert f(cq=_cu(1, 4)) == INVALID and f(cq=_cu(0, 4, 3), ck=_cu(0, 8, 8), nseg=2) == INVALID
        assert f(nseg=0) == INVALID
        assert f(cq=_cu(*range(66)), ck=_cu(*range(66)), nseg=65) == UNSUPPORTED
        assert f(h=2048, hk=1, **({} if f is size else dict(ldq=1 << 17))) == UNSUPPORTED
        assert f(cq=_cu(0, 1 << 30)) == UNSUPPORTED  # 2^31 rows
    assert size(out=None) == INVALID
    assert call(ldq=120) == INVALID and call(ldq=132) == INVALID
    assert call(kl=_cu(9)) == INVALID and call(kl=_cu(-1)) == INVALID
    for kw in (dict(q=None), dict(o=None), dict(c=None), dict(ws=None), dict(q=258), dict(o=8), dict(c=24),
               dict(ws=128)):
        assert call(**kw) == INVALID, kw
    assert call(nbytes=need.value - 1) == WORKSPACE
    assert call(have=2 * 64 * 64 + 255) == WORKSPACE
    assert call(cq=_cu(0, 0), q=None, o=None, c=None, ws=None, nbytes=0) == OK  # no queries


def test_refine_refusals(L):
    P = ctypes.c_void_p
    reqs = S.make_requests([W.Request(2, 8, 8)])
    n, m = ctypes.c_size_t(), ctypes.c_size_t()
    tiny = S.model_desc(W.TINY_MODEL, 256)  # head_dim 16
    assert L.sphinx_kv8_cache_bytes(ctypes.byref(tiny), reqs, 1, ctypes.byref(n)) == UNSUPPORTED
    assert L.sphinx_refine_kv8_workspace_bytes(ctypes.byref(tiny), reqs, 1, 5, ctypes.byref(n)) == UNSUPPORTED
    d = S.model_desc(W.SMALL_MODEL, 256)
    assert L.sphinx_kv8_cache_bytes(ctypes.byref(d), reqs, 1, ctypes.byref(n)) == OK
    assert n.value == W.SMALL_MODEL.L * S.sphinx_kv8_bytes(W.SMALL_MODEL.heads, 64, [0, 32])
    assert L.sphinx_kv8_cache_bytes(ctypes.byref(d), reqs, 1, None) == INVALID
    assert L.sphinx_refine_kv8_workspace_bytes(ctypes.byref(d), reqs, 1, 40, ctypes.byref(m)) == INVALID
    assert L.sphinx_refine_kv8_workspace_bytes(ctypes.byref(d), reqs, 1, 5, ctypes.byref(m)) == OK
    assert m.value > S.sphinx_refine_workspace_bytes(d, reqs, 5)
    args = lambda desc, cache, nbytes: (ctypes.byref(desc), reqs, 1, P(256), 5, _cu(0, 5), P(256), P(256), P(256),
                                        P(256), P(cache), P(256), nbytes, None)
    assert L.sphinx_refine_step_kv8(*args(d, 256, m.value - 1)) == WORKSPACE
    assert L.sphinx_refine_step_kv8(*args(d, None, m.value)) == INVALID
    assert L.sphinx_refine_step_kv8(*args(d, 264, m.value)) == INVALID
    assert L.sphinx_refine_step_kv8(*args(tiny, 256, 1 << 40)) == UNSUPPORTED
