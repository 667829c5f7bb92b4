"""The 8-bit key/value cache through the C ABI against its float64 oracle: rows
written and read back bit for bit, attention over the cache within rounding
bounds, and the refinement step that uses both."""
import numpy as np
import pytest

import oracle as O
import workloads as W

torch = pytest.importorskip("torch")
S = pytest.importorskip("paper_2511_18672_amd")
B = S.binding

pytestmark = pytest.mark.gpu

TDT = {"f32": torch.float32, "bf16": torch.bfloat16}
BOUNDS = {"one": [0, 1], "block": [0, 64], "odd": [0, 65, 65, 66, 257], "many": [0, 63, 191, 1000, 1001, 1130]}


def say(*a):
    print(*a, flush=True)


def rows_of(rng, n, heads, d, dtype):
    """Random rows as tensors of the type, with sizes that vary from row to row."""
    x = rng.standard_normal((n, heads, d)) * np.exp2(rng.integers(-6, 7, (n, 1, 1)))
    return torch.from_numpy(x.astype(np.float32)).to(TDT[dtype]).cuda()


def f64(t):
    return t.double().cpu().numpy()


class Cache:
    """A slice with its bounds, and what the oracle says it holds."""

    def __init__(self, heads, d, bounds, fill=0):
        self.heads, self.d, self.bounds, self.n = heads, d, np.asarray(bounds, np.int32), int(bounds[-1])
        self.slice = torch.full((B.sphinx_kv8_bytes(heads, d, bounds),), fill, dtype=torch.uint8, device="cuda")
        self.k = np.zeros((self.n, heads, d))
        self.v = np.zeros((self.n, heads, d))

    def store(self, k, v, idx=None, ld=None, stream=None):
        n, dtype = k.shape[0], B.F32 if k.dtype == torch.float32 else B.BF16
        ld = ld or k.stride(0)
        i = None if idx is None else torch.as_tensor(np.asarray(idx, np.int32)).cuda()
        B.sphinx_kv8_store(dtype, self.heads, self.d, k, v, ld, i, n, self.bounds, self.slice, stream)
        at = np.arange(n) if idx is None else np.asarray(idx)
        self.k = O.kv8.write(self.k, f64(k).reshape(n, self.heads, self.d), at, self.bounds)
        self.v = O.kv8.write(self.v, f64(v).reshape(n, self.heads, self.d), at, self.bounds)

    def load(self, dtype="f32", idx=None, n=None, pad=0):
        n = self.n if idx is None and n is None else (n if idx is None else len(idx))
        w = self.heads * self.d
        k = torch.full((n, w + pad), 7.0, dtype=TDT[dtype], device="cuda")
        v = torch.full((n, w + pad), 7.0, dtype=TDT[dtype], device="cuda")
        i = None if idx is None else torch.as_tensor(np.asarray(idx, np.int32)).cuda()
        B.sphinx_kv8_load(B.F32 if dtype == "f32" else B.BF16, self.heads, self.d, self.slice, self.bounds, i, n, k, v,
                          w + pad)
        return k, v

    def check(self, dtype="f32"):
        k, v = self.load(dtype)
        shape = (self.n, self.heads, self.d)
        assert np.array_equal(f64(k).reshape(shape), self.k, equal_nan=True)
        assert np.array_equal(f64(v).reshape(shape), self.v, equal_nan=True)


# ---------------------------------------------------------------------------
# writing and reading back
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("bounds", list(BOUNDS))
@pytest.mark.parametrize("heads,d", [(1, 64), (3, 72), (4, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_store_all_then_some(dtype, heads, d, bounds):
    say(f"[kv8 store] {dtype} heads {heads} d {d} bounds {BOUNDS[bounds]}")
    rng = np.random.default_rng(5)
    c = Cache(heads, d, BOUNDS[bounds])
    c.store(rows_of(rng, c.n, heads, d, dtype), rows_of(rng, c.n, heads, d, dtype))
    c.check(dtype)
    idx = np.flatnonzero(rng.random(c.n) < 0.3)
    # larger and smaller rows than before: the scales of the touched blocks grow and shrink
    for size in (300.0, 1.0 / 64.0):
        k, v = (rows_of(rng, idx.size, heads, d, dtype) * size for _ in range(2))
        c.store(k, v, idx)
        c.check("f32")


def test_store_a_prefix_and_strided_columns():
    rng = np.random.default_rng(6)
    c = Cache(2, 64, [0, 100, 300])
    both = rows_of(rng, 170, 6, 64, "bf16").view(170, 384)  # keys in columns 128 .. 255, values behind them
    c.store(both[:, 128:256].unflatten(1, (2, 64)), both[:, 256:].unflatten(1, (2, 64)), ld=384)
    c.check()
    k, _ = c.load("bf16", pad=24)
    assert (k[:, 128:] == 7.0).all()
    k, _ = c.load("bf16", n=70)
    assert np.array_equal(f64(k).reshape(70, 2, 64), c.k[:70])


def test_store_repeated_and_outside_tokens():
    rng = np.random.default_rng(7)
    c = Cache(2, 72, [0, 130, 200])
    c.store(rows_of(rng, 200, 2, 72, "bf16"), rows_of(rng, 200, 2, 72, "bf16"))
    idx = [-5, -1, 3, 3, 3, 63, 64, 64, 129, 130, 199, 200, 1 << 30]
    c.store(rows_of(rng, len(idx), 2, 72, "bf16"), rows_of(rng, len(idx), 2, 72, "bf16"), idx)
    c.check()
    many = [70] * 150 + [71] * 70  # one block named by more rows than it has
    c.store(rows_of(rng, 220, 2, 72, "bf16"), rows_of(rng, 220, 2, 72, "bf16"), many)
    c.check()
    say("[kv8 load] repeated and outside tokens")
    k, v = c.load("f32", idx)
    got = f64(k).reshape(-1, 2, 72)
    for j, t in enumerate(idx):
        want = c.k[t] if 0 <= t < 200 else np.full((2, 72), 7.0)
        assert np.array_equal(got[j], want), t
    k, _ = c.load("bf16", many)
    assert np.array_equal(f64(k).reshape(-1, 2, 72), c.k[many])


def test_store_of_what_8_bits_cannot_hold():
    """Zeros, subnormals, the largest floats, infinities and NaN."""
    c = Cache(1, 64, [0, 64, 128, 192, 256, 320])
    x = torch.zeros(320, 1, 64)
    x[64:128] = torch.randn(64, 1, 64) * 1e-41
    x[128:192] = torch.randn(64, 1, 64).clamp(-1, 1) * 3.4e38
    x[192:256] = torch.randn(64, 1, 64)
    x[192, 0, :3] = torch.tensor([float("inf"), -float("inf"), float("nan")])
    x[256:320] = float("inf")
    x = x.cuda()
    c.store(x, -x)
    c.check("f32")
    bf = x.bfloat16()
    c.store(bf, -bf)
    c.check("bf16")
    # a block of NaN and infinities takes ordinary rows again
    y = torch.randn(64, 1, 64, device="cuda")
    c.store(y, y, np.arange(256, 320))
    c.check("f32")


def test_a_slice_of_any_bytes_written_whole():
    """Nothing that an uncleared slice held survives in blocks written whole."""
    rng = np.random.default_rng(8)
    for fill in (0xFF, 0x7F, 0x80):
        c = Cache(2, 72, [0, 64, 192], fill)
        c.store(rows_of(rng, 192, 2, 72, "bf16"), rows_of(rng, 192, 2, 72, "bf16"))
        c.check()


@pytest.mark.parametrize("idx", [np.arange(300), np.arange(7, 290), np.r_[0:64, 63, 64:128], np.r_[-3, 0:128, 128, 128],
                                 np.r_[0:32, 32:64, 128:192, 200:300], np.r_[0, 0, 2:64, 64:300]],
                         ids=["all", "inner", "one_twice", "last_twice", "blocks", "gap_and_twice"])
@pytest.mark.parametrize("bounds", [[0, 300], [0, 64, 130, 300], [0, 63, 300]])
def test_listed_whole_blocks(idx, bounds):
    """Runs that fill a block, that fill it and list a token again, that only seem to."""
    rng = np.random.default_rng(11)
    c = Cache(3, 72, bounds)
    c.store(rows_of(rng, 300, 3, 72, "bf16"), rows_of(rng, 300, 3, 72, "bf16"))
    c.store(rows_of(rng, idx.size, 3, 72, "bf16"), rows_of(rng, idx.size, 3, 72, "bf16"), idx)
    c.check("bf16")
    k, v = c.load("f32", idx)
    inside = idx >= 0
    assert np.array_equal(f64(k).reshape(-1, 3, 72)[inside], c.k[idx[inside]])
    assert np.array_equal(f64(v).reshape(-1, 3, 72)[inside], c.v[idx[inside]])


@pytest.mark.parametrize("heads,d", [(32, 64), (24, 72)])
def test_many_listed_rows_of_many_heads(heads, d):
    """Enough rows that a worker looks at 32 of them (storing) and at 64 (reading back): whole blocks, runs that start
    and end anywhere, single and repeated tokens, tokens in front of the slice and behind it."""
    rng = np.random.default_rng(13)
    bounds = [0, 1000, 1001, 4097, 7000]
    some = np.flatnonzero(np.repeat(rng.random(1001) < 0.4, 7)[:7000])
    runs = np.r_[0:64, 70:200, 1000:1001, 1001:1193, 1200:1264, 1265:4097, 4097:4161, 4170:6990]
    c = Cache(heads, d, bounds)
    k, v = (torch.randn(7000, heads * d, device="cuda").bfloat16() for _ in range(2))
    c.store(k, v, np.arange(7000))
    for idx in (runs, np.r_[-2, -1, np.repeat(some, 1 + (rng.random(some.size) < 0.1)), 7000, 7003]):
        n = len(idx)
        k, v = (torch.randn(n, heads * d, device="cuda").bfloat16() * 3 for _ in range(2))
        keep = (idx >= 0) & (idx < 7000)
        i = torch.from_numpy(idx.astype(np.int32)).cuda()
        B.sphinx_kv8_store(B.BF16, heads, d, k, v, heads * d, i, n, bounds, c.slice)
        for name, x in (("k", k), ("v", v)):  # the last of repeated tokens counts, as numpy assigns
            setattr(c, name, O.kv8.write(getattr(c, name), f64(x).reshape(n, heads, d)[keep], idx[keep], bounds))
        c.check("bf16")
        ko, vo = c.load("bf16", idx)
        for out, held in ((ko, c.k), (vo, c.v)):
            assert np.array_equal(f64(out)[keep].reshape(-1, heads, d), held[idx[keep]])
            assert (out[torch.from_numpy(~keep).cuda()] == 7).all()


def test_load_some_rows():
    rng = np.random.default_rng(9)
    for heads, d, dtype in ((3, 64, "f32"), (2, 72, "bf16")):
        c = Cache(heads, d, [0, 700, 701, 1500])
        c.store(rows_of(rng, 1500, heads, d, "bf16"), rows_of(rng, 1500, heads, d, "bf16"))
        for idx in ([0], [699, 700, 701], np.flatnonzero(rng.random(1500) < 0.4)):
            k, v = c.load(dtype, idx)
            assert np.array_equal(f64(k).reshape(-1, heads, d), c.k[idx])
            assert np.array_equal(f64(v).reshape(-1, heads, d), c.v[idx])


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def tolerance(dtype, ref, mag, big, keys, d):
    """Bound of |o - ref| by roundings.  A score is off by at most d roundings of fp32 sums relative to sum |q k|; the
    exponential, sums and products of weights by 2^-22 and `keys` fp32 roundings more (each a factor on weights whose
    weighted |v| is `mag`, once in the numerator and once in the denominator); bf16 weights by 2^-8 in each; the result
    rounds once."""
    w = np.log(2.0) * (d + 2) * 2.0 ** -24 * big + 2.0 ** -22 + (keys + 8) * 2.0 ** -24
    if dtype == "bf16":
        return 2.02 * (w + 2.0 ** -8) * mag + 2.0 ** -8 * np.abs(ref) + 1e-30
    return 2.02 * w * mag + 2.0 ** -24 * np.abs(ref) + 1e-30


def attend(c, q, heads, cu_q, kv_len=None, ldq=None, stream=None, out=None, ws=None):
    dtype = B.F32 if q.dtype == torch.float32 else B.BF16
    o = torch.full((q.shape[0], heads * c.d), 7.0, dtype=q.dtype, device="cuda") if out is None else out
    need = B.sphinx_kv8_attention_workspace_bytes(dtype, heads, c.heads, c.d, cu_q, c.bounds)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda") if ws is None else ws
    B.sphinx_kv8_attention(dtype, heads, c.heads, c.d, q, ldq or heads * c.d, c.slice, c.bounds, kv_len, o, cu_q, ws,
                           stream)
    return o


def check_attention(c, q, heads, cu_q, kv_len=None, **kw):
    dtype = "f32" if q.dtype == torch.float32 else "bf16"
    o = f64(attend(c, q, heads, cu_q, kv_len, **kw)).reshape(-1, heads, c.d)
    qq = f64(q)[:, :heads * c.d].reshape(-1, heads, c.d)
    ref, mag, big = O.kv8.attention(qq, c.k, c.v, cu_q, c.bounds, kv_len)
    keys = int(np.diff(c.bounds).max()) if kv_len is None else max(kv_len)
    n = int(cu_q[-1])
    err = np.abs(o[:n] - ref[:n]) - tolerance(dtype, ref[:n], mag[:n], big[:n], keys, c.d)
    say(f"[kv8 attention] {dtype} heads {heads}/{c.heads} d {c.d} max_abs {np.abs(o[:n] - ref[:n]).max():.3e} "
        f"over bound {err.max():.3e}")
    assert np.isfinite(o[:n]).all() and err.max() <= 0.0
    assert (o[n:] == 7.0).all()  # rows behind the last query
    return o


def filled(rng, heads, d, bounds, dtype="bf16", fill=0, strong=3.0):
    c = Cache(heads, d, bounds, fill)
    k, v = rows_of(rng, c.n, heads, d, dtype), rows_of(rng, c.n, heads, d, dtype)
    if c.n:
        c.store(torch.randn_like(k) * strong, v)
    return c


def queries(rng, n, heads, d, dtype):
    q = rng.standard_normal((n, heads * d)) * (np.log2(np.e) / np.sqrt(d))
    return torch.from_numpy(q.astype(np.float32)).to(TDT[dtype]).cuda()


SEGMENTS = [([1], [1]), ([1], [64]), ([3], [65]), ([32], [63]), ([33], [200]), ([129], [640]),
            ([1, 0, 5, 40], [700, 30, 1, 129]), ([257, 1, 64], [97, 1025, 64])]


@pytest.mark.parametrize("kind", [("bf16", 64, 1, 1), ("bf16", 64, 2, 4), ("bf16", 72, 3, 1), ("bf16", 72, 1, 5),
                                  ("f32", 64, 2, 1), ("f32", 64, 1, 3)])
@pytest.mark.parametrize("seg", range(len(SEGMENTS)))
def test_attention_sizes(seg, kind):
    dtype, d, kv_heads, group = kind
    nq, nk = SEGMENTS[seg]
    rng = np.random.default_rng(10 + seg)
    c = filled(rng, kv_heads, d, np.concatenate([[0], np.cumsum(nk)]), dtype)
    cu_q = np.concatenate([[0], np.cumsum(nq)])
    q = queries(rng, cu_q[-1] + 2, kv_heads * group, d, dtype)
    check_attention(c, q, kv_heads * group, cu_q)


@pytest.mark.parametrize("dtype,d,nq,nk", [("bf16", 64, 1, 9000), ("bf16", 64, 5, 20001), ("bf16", 72, 2, 12345),
                                           ("f32", 64, 1, 9001), ("bf16", 64, 700, 3001), ("bf16", 72, 515, 2500),
                                           ("f32", 64, 130, 2500)])
def test_attention_long(dtype, d, nq, nk):
    rng = np.random.default_rng(20)
    c = filled(rng, 2, d, [0, nk], dtype)
    check_attention(c, queries(rng, nq, 2, d, dtype), 2, [0, nq])


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 72), ("f32", 64)])
@pytest.mark.parametrize("nq", [2, 300])
def test_attention_looks_at_kv_len_tokens_only(dtype, d, nq):
    """Behind kv_len the slice holds NaN (bytes 0xFF) or other rows; a segment without keys gives zeros."""
    rng = np.random.default_rng(21)
    bounds = [0, 300, 500, 600, 1700]
    c = Cache(2, d, bounds, fill=0xFF)
    c.k[:], c.v[:] = np.nan, np.nan
    lens = [70, 200, 0, 1029]
    idx = np.concatenate([np.arange(b, b + n) for b, n in zip(bounds, lens)])
    k, v = rows_of(rng, idx.size, 2, d, dtype), rows_of(rng, idx.size, 2, d, dtype)
    c.store(k / 8, v, idx)
    q = queries(rng, 4 * nq, 4, d, dtype)
    o = check_attention(c, q, 4, np.arange(5) * nq, lens)
    assert (o[2 * nq:3 * nq] == 0.0).all()


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 72), ("f32", 64)])
@pytest.mark.parametrize("nq", [1, 150])
@pytest.mark.parametrize("size,shift", [(1.0, 2000.0), (40.0, 0.0), (1.0, -2000.0), (1e-3, 0.0)])
def test_attention_of_large_and_small_scores(dtype, d, nq, size, shift):
    """Scores spread over +-1000, or all near +-2000, or all near 0: the softmax neither overflows nor vanishes."""
    rng = np.random.default_rng(22)
    nk = 777
    c = Cache(1, d, [0, nk])
    k = rows_of(rng, nk, 1, d, dtype) * 0 + torch.randn(nk, 1, d, device="cuda", dtype=TDT[dtype]) * size
    k[:, :, 0] = 8.0
    # the scores grow along the keys, so that the running maximum moves again and again
    k[:, 0, 1] = torch.linspace(-4, 4, nk, device="cuda").to(k.dtype)
    c.store(k, rows_of(rng, nk, 1, d, dtype))
    q = queries(rng, nq, 1, d, dtype) * 4.0
    q[:, 0] = shift / 8.0
    q[:, 1] = 30.0
    check_attention(c, q, 1, [0, nq])


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 72), ("f32", 64)])
@pytest.mark.parametrize("nq", [1, 300])
@pytest.mark.parametrize("low", [-(2.0 ** 100), -(2.0 ** 127)])
@pytest.mark.parametrize("at", [0, 64, 320])
def test_attention_of_a_block_whose_scores_are_far_below(dtype, d, nq, low, at):
    """One block's scores are about -2^101 or past f32's range (-inf), all others of a row -192, -208 or -224: what a
    score is taken relative to moves between them exactly, wherever that block stands."""
    rng = np.random.default_rng(33)
    nk = 400
    c = Cache(1, d, [0, nk])
    k = torch.zeros(nk, 1, d)
    k[:, 0, 0] = torch.tensor([-192.0, -208.0, -224.0])[torch.arange(nk) % 3] / 2  # exact in 8 bits
    k[at:at + 64, 0, 0] = low
    v = rows_of(rng, nk, 1, d, dtype)
    c.store(k.to(TDT[dtype]).cuda(), v)
    q = torch.zeros(nq, d, dtype=TDT[dtype], device="cuda")
    q[:, 0] = 2.0
    assert (c.k[at:at + 64, 0, 0] == low).all() and c.k[(at + 64) % nk, 0, 0] > -113.0
    ref, mag, _ = O.kv8.attention(f64(q).reshape(nq, 1, d), c.k, c.v, [0, nq], c.bounds)
    o = f64(attend(c, q, 1, [0, nq])).reshape(nq, 1, d)
    # the scores that weigh are exact
    err = np.abs(o - ref) - tolerance(dtype, ref, mag, np.zeros_like(mag), nk, d)
    assert np.isfinite(o).all() and err.max() <= 0.0


def test_attention_strided_queries():
    rng = np.random.default_rng(23)
    c = filled(rng, 2, 64, [0, 300])
    for nq in (3, 200):
        q = queries(rng, nq, 9, 64, "bf16")  # rows of 576, the first 256 columns are the queries
        o = attend(c, q, 4, [0, nq], ldq=576)
        p = attend(c, q[:, :256].contiguous(), 4, [0, nq])
        assert torch.equal(o, p)


def test_attention_nan_key_reaches_its_queries_only():
    rng = np.random.default_rng(24)
    for nq in (2, 140):
        c = Cache(2, 64, [0, 100, 300])
        k, v = rows_of(rng, 300, 2, 64, "bf16"), rows_of(rng, 300, 2, 64, "bf16")
        k[50, 1, 3] = float("nan")
        c.store(k, v)
        q = queries(rng, 2 * nq, 2, 64, "bf16")
        o = attend(c, q, 2, [0, nq, 2 * nq]).view(2 * nq, 2, 64)
        assert torch.isnan(o[:nq, 1]).all() and torch.isfinite(o[:nq, 0]).all() and torch.isfinite(o[nq:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kv_heads,group,nq,nk", [(1, 96, 3, 500), (1, 512, 1, 100), (40, 1, 2, 70), (3, 7, 33, 129)])
def test_attention_head_layouts(dtype, kv_heads, group, nq, nk):
    rng = np.random.default_rng(28)
    c = filled(rng, kv_heads, 64, [0, nk], dtype)
    check_attention(c, queries(rng, nq, kv_heads * group, 64, dtype), kv_heads * group, [0, nq])


def test_attention_of_64_segments():
    """The most segments of a call, some without queries, some without keys, in blocks of every fill."""
    rng = np.random.default_rng(29)
    for scale in (1, 5):
        nk = rng.integers(0, 300 * scale, 64)
        nq = rng.integers(0, 3 * scale * scale, 64)
        nk[[3, 40]], nq[[4, 41]], nk[63], nq[63] = 0, 0, 64, 2
        c = filled(rng, 2, 72, np.concatenate([[0], np.cumsum(nk)]))
        cu_q = np.concatenate([[0], np.cumsum(nq)])
        check_attention(c, queries(rng, cu_q[-1], 6, 72, "bf16"), 6, cu_q)


@pytest.mark.parametrize("nq", [1, 40, 300])
def test_attention_over_a_cleared_slice_is_zero(nq):
    c = Cache(2, 72, [0, 1000])
    q = queries(np.random.default_rng(30), nq, 2, 72, "bf16")
    assert (attend(c, q, 2, [0, nq]) == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nq", [5, 140])
def test_attention_of_a_nan_or_infinite_query_leaves_the_others(dtype, nq):
    rng = np.random.default_rng(31)
    c = filled(rng, 2, 64, [0, 400], dtype)
    q = queries(rng, nq, 2, 64, dtype)
    q[1, 5] = float("nan")
    q[3, 70] = float("inf")
    o = f64(attend(c, q, 2, [0, nq])).reshape(nq, 2, 64)
    assert np.isnan(o[1, 0]).all() and np.isnan(o[3, 1]).all()
    qq = f64(q).reshape(nq, 2, 64)
    qq[1, 0], qq[3, 1] = 0.0, 0.0
    ref, mag, big = O.kv8.attention(qq, c.k, c.v, [0, nq], c.bounds)
    err = np.abs(o - ref) - tolerance(dtype, ref, mag, big, 400, 64)
    err[1, 0], err[3, 1] = -1.0, -1.0
    assert err.max() <= 0.0


def test_slice_at_any_16_bytes():
    """A slice needs no more than 16-byte alignment."""
    rng = np.random.default_rng(32)
    c = Cache(3, 72, [0, 200])
    whole = torch.zeros(c.slice.numel() + 64, dtype=torch.uint8, device="cuda")
    c.slice = whole[48:48 + c.slice.numel()]
    c.store(rows_of(rng, 200, 3, 72, "bf16"), rows_of(rng, 200, 3, 72, "bf16"))
    c.check("bf16")
    for nq in (2, 200):
        check_attention(c, queries(rng, nq, 3, 72, "bf16"), 3, [0, nq])
    assert (whole[:48] == 0).all() and (whole[48 + c.slice.numel():] == 0).all()


@pytest.mark.parametrize("nq,nk", [(1, 8000), (400, 4000)])
def test_attention_repeats_bit_for_bit_on_streams_and_in_graphs(nq, nk):
    rng = np.random.default_rng(25)
    c = filled(rng, 4, 64, [0, nk, nk + 70])
    cu_q = [0, nq, nq + 3]
    q = queries(rng, nq + 3, 8, 64, "bf16")
    first = attend(c, q, 8, cu_q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    second = attend(c, q, 8, cu_q, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(first, second)
    # a captured store and attention, replayed between eager work on the same cache
    k, v = rows_of(rng, 40, 4, 64, "bf16"), rows_of(rng, 40, 4, 64, "bf16")
    idx = torch.arange(10, 50, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.sphinx_kv8_attention_workspace_bytes(B.BF16, 8, 4, 64, cu_q, c.bounds), dtype=torch.uint8,
                     device="cuda")
    o = torch.empty_like(first)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        B.sphinx_kv8_store(B.BF16, 4, 64, k, v, 256, idx, 40, c.bounds, c.slice)
        attend(c, q, 8, cu_q, out=o, ws=ws)
    for i in range(3):
        k.normal_()
        q.mul_(0.9)
        g.replay()
        torch.cuda.synchronize()
        want = Cache(4, 64, c.bounds)
        want.slice.copy_(c.slice)
        B.sphinx_kv8_store(B.BF16, 4, 64, k, v, 256, idx, 40, c.bounds, want.slice)
        assert torch.equal(want.slice, c.slice), i
        assert torch.equal(attend(want, q, 8, cu_q), o), i


def test_segments_do_not_depend_on_what_they_are_packed_with():
    """What a segment's part of the cache holds is the same alone and packed."""
    rng = np.random.default_rng(26)
    k, v = rows_of(rng, 500, 2, 64, "bf16"), rows_of(rng, 500, 2, 64, "bf16")
    both = Cache(2, 64, [0, 230, 500])
    both.store(k, v)
    alone = Cache(2, 64, [0, 270])
    alone.store(k[230:], v[230:])
    assert torch.equal(both.load("bf16")[0][230:], alone.load("bf16")[0])


def test_cache_past_32_bit_offsets():
    """2^23 + 100 tokens of five heads: 5.4 GB.  All but a few rows are zero, so a zero key weighs 2^0 and adds nothing;
    the rows at the far end of the last head lie past 4 GB."""
    n, heads = (1 << 23) + 100, 5
    rng = np.random.default_rng(27)
    size = B.sphinx_kv8_bytes(heads, 64, [0, n])
    assert size > 1 << 32
    cache = torch.zeros(size, dtype=torch.uint8, device="cuda")
    idx = np.array([0, 1 << 22, n - 70, n - 2, n - 1], np.int32)
    k, v = (rng.standard_normal((5, heads, 64)) for _ in range(2))
    k, v = (torch.from_numpy(x.astype(np.float32)).bfloat16().cuda() for x in (k * 4, v * 1e6))
    ii = torch.from_numpy(idx).cuda()
    B.sphinx_kv8_store(B.BF16, heads, 64, k, v, heads * 64, ii, 5, [0, n], cache)
    k2, v2 = torch.empty(5, heads, 64, device="cuda"), torch.empty(5, heads, 64, device="cuda")
    B.sphinx_kv8_load(B.F32, heads, 64, cache, [0, n], ii, 5, k2, v2, heads * 64)
    # rows 3 and 4 share a block
    bounds = [0, 1, 2, 3, 5]
    K, V = O.kv8.quantise(f64(k), bounds), O.kv8.quantise(f64(v), bounds)
    assert np.array_equal(f64(k2), K) and np.array_equal(f64(v2), V)
    for nq in (1, 40):
        q = queries(rng, nq, heads, 64, "bf16") * 3
        o = torch.empty(nq, heads * 64, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(B.sphinx_kv8_attention_workspace_bytes(B.BF16, heads, heads, 64, [0, nq], [0, n]),
                         dtype=torch.uint8, device="cuda")
        B.sphinx_kv8_attention(B.BF16, heads, heads, 64, q, heads * 64, cache, [0, n], None, o, [0, nq], ws)
        w = np.exp2(np.einsum("qhd,thd->qht", f64(q).reshape(nq, heads, 64), K))
        den = w.sum(2) + (n - 5)
        ref = np.einsum("qht,thd->qhd", w, V) / den[..., None]
        mag = np.einsum("qht,thd->qhd", w, np.abs(V)) / den[..., None]
        # fp32 sums of 2^23 equal numbers, added in runs of at most 2^17 blocks: 2^-7 covers their roundings
        err = np.abs(f64(o).reshape(nq, heads, 64) - ref)
        assert (err <= mag * 2.0 ** -6 + 2.0 ** -8 * np.abs(ref)).all()


def test_tensors_of_another_device_and_short_slices_are_refused():
    c = Cache(1, 64, [0, 64])
    cpu = torch.zeros(64, 64)
    with pytest.raises(ValueError):
        B.sphinx_kv8_store(B.F32, 1, 64, cpu, cpu, 64, None, 64, c.bounds, c.slice)
    rows = torch.zeros(64, 64, device="cuda")
    for idx in (torch.arange(64, device="cuda"), torch.arange(63, dtype=torch.int32, device="cuda")):  # int64; too few
        with pytest.raises(ValueError):
            B.sphinx_kv8_store(B.F32, 1, 64, rows, rows, 64, idx, 64, c.bounds, c.slice)
        with pytest.raises(ValueError):
            B.sphinx_kv8_load(B.F32, 1, 64, c.slice, c.bounds, idx, 64, rows, rows, 64)
    with pytest.raises(S.SphinxError):  # a slice of too few bytes
        B.sphinx_kv8_load(B.F32, 1, 64, c.slice[:64], c.bounds, None, 64, cpu.cuda(), cpu.cuda(), 64)


# ---------------------------------------------------------------------------
# the refinement step with the 8-bit cache
# ---------------------------------------------------------------------------
MID = dict(mlp=512, L=2)
MODELS = {
    "bf16_64": W.ModelCfg(D=128, heads=2, head_dim=64, dtype="bf16", **MID),
    "bf16_72": W.ModelCfg(D=1152, heads=16, head_dim=72, mlp=1152, L=1, dtype="bf16"),
    "f32_64": W.ModelCfg(D=128, heads=2, head_dim=64, dtype="f32", **MID),
    "factorised": W.ModelCfg(D=128, heads=2, head_dim=64, dtype="bf16", attention="factorised", **MID),
}


@pytest.mark.parametrize("model", list(MODELS))
@pytest.mark.parametrize("period", [2, 3])
def test_refine_with_the_8_bit_cache(model, period):
    """The whole loop against the oracle whose cache holds the same 8-bit numbers, to the framework's bounds for latents
    (2e-2 for bf16 models).  An fp32 model differs from the oracle only where a key or value lies so near the middle of
    two 8-bit numbers that fp32 rounding decides: one step is 2^-3 of the value for one of 64 dims of one key, so its
    latents are held to the same bound, not to the 1e-4 of an unrounded cache."""
    cfg = MODELS[model]
    shapes = [W.Request(4, 16, 16)] if model == "bf16_72" else [W.Request(3, 24, 20), W.Request(2, 10, 14),
                                                                 W.Request(1, 4, 4)]
    n = len(shapes)
    wl = W.custom("kv8_" + model, cfg, shapes, [0.4, 0.7, 0.5][:n], [("uniform", 0.3, 0.7), 0.5, 0.2][:n],
                  [5, 4, 3][:n])
    R = S.from_workload(wl, cache_period=period, cache_dtype="fp8")
    got = R.run().cpu().numpy().astype(np.float64)
    ref = O.refine(wl, precision="model", period=period, cache8=True)
    plain = O.refine(wl, precision="model", period=period)
    err = np.abs(got - ref).max()
    say(f"[kv8 refine {model} T={period}] max_abs {err:.3e} (8-bit against unrounded cache: "
        f"{np.abs(plain - ref).max():.3e})")
    assert np.isfinite(got).all() and err <= 2e-2


def test_refine_with_the_8_bit_cache_repeats_and_keeps_unselected_tokens():
    wl = W.custom("kv8_repeat", W.ModelCfg(D=1024, heads=16, head_dim=64, mlp=4096, L=2, dtype="bf16"),
                  [W.Request(14, 32, 64)], [0.3], [0.5], [3])
    outs = []
    for _ in range(2):
        R = S.from_workload(wl, cache_period=3, cache_dtype="fp8")
        R.reset()
        for i in range(3):
            n = R.step(i)
        outs.append(R.state.cpu().numpy())
        idx = R.idx[:n].cpu().numpy()
    assert np.array_equal(outs[0], outs[1]) and np.isfinite(outs[0]).all()
    keep = np.ones(wl.N, bool)
    keep[idx] = False
    P = O.patchify(outs[0], wl.requests)
    assert np.array_equal(P[keep], O.patchify(wl.z0, wl.requests)[keep].astype(np.float32))


def test_refiner_refuses_a_cache_type_without_a_cache():
    wl = W.custom("kv8_args", MODELS["bf16_64"], [W.Request(1, 8, 8)], [0.5], [0.5], [1])
    with pytest.raises(ValueError):
        S.from_workload(wl, cache_dtype="fp8")
    with pytest.raises(ValueError):
        S.from_workload(wl, cache_period=2, cache_dtype="int8")
