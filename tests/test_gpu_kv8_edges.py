"""The 8-bit key/value cache through the C ABI where it can go wrong: sums that overflow late in a block, weights that
bf16 misses, segments packed and alone, a slice that is used again, offsets past 32 bits."""
import numpy as np
import pytest

import oracle as O

torch = pytest.importorskip("torch")
S = pytest.importorskip("paper_2511_18672_amd")
B = S.binding

from test_gpu_kv8 import TDT, Cache, attend, check_attention, f64, filled, queries, rows_of, tolerance  # noqa: E402
from test_kv8_rules import plan  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 72), ("f32", 64)])
@pytest.mark.parametrize("nq", [1, 300])
@pytest.mark.parametrize("score", [34.0, 192.0])
def test_one_late_key_of_a_block_that_outweighs_all_others(dtype, d, nq, score):
    """Scores are 0 but for one token's: 2^192 is past f32's range, 2^34 only past what a block's weights may sum to.
    The tokens are those whose weights are added last, in a block in front of others and in a segment's last one."""
    rng = np.random.default_rng(41)
    for t in (58, 59, 62, 63):
        for at in (64 + t, 5 * 64 + t):
            c = Cache(1, d, [0, 384])
            k = torch.zeros(384, 1, d)
            k[at, 0, 0] = 32.0 if score < 100 else 192.0  # exact in 8 bits
            c.store(k.to(TDT[dtype]).cuda(), rows_of(rng, 384, 1, d, dtype))
            q = torch.zeros(nq, d, dtype=TDT[dtype], device="cuda")
            q[:, 0] = score / float(k[at, 0, 0])
            ref, mag, _ = O.kv8.attention(f64(q).reshape(nq, 1, d), c.k, c.v, [0, nq], c.bounds)
            o = f64(attend(c, q, 1, [0, nq])).reshape(nq, 1, d)
            err = np.abs(o - ref) - tolerance(dtype, ref, mag, np.zeros_like(mag), 384, d)  # scores are exact
            assert np.isfinite(o).all() and err.max() <= 0.0, (t, at)


@pytest.mark.parametrize("d", [64, 72])
@pytest.mark.parametrize("score", [66.0, 192.0])
def test_one_late_key_of_a_block_in_16_bit_attention(d, score):
    """The same through sphinx_varlen_attention."""
    rng = np.random.default_rng(42)
    v = rows_of(rng, 384, 1, d, "bf16").view(384, d)
    q = torch.zeros(300, d, dtype=torch.bfloat16, device="cuda")
    q[:, 0] = 1.0
    for t in range(50, 64):
        for at in (64 + t, 5 * 64 + t):
            k = torch.zeros(384, d, dtype=torch.bfloat16, device="cuda")
            k[at, 0] = score
            o = torch.empty_like(q)
            B.sphinx_varlen_attention(B.BF16, 1, d, q, d, k, v, d, o, [0, 300], [0, 384])
            shape = (-1, 1, d)
            ref, mag, _ = O.kv8.attention(f64(q).reshape(shape), f64(k).reshape(shape), f64(v).reshape(shape), [0, 300],
                                          [0, 384])
            o = f64(o).reshape(shape)
            err = np.abs(o - ref) - tolerance("bf16", ref, mag, np.zeros_like(mag), 384, d)
            assert np.isfinite(o).all() and err.max() <= 0.0, (t, at)


@pytest.mark.parametrize("d,nq,nk", [(64, 1, 512), (64, 40, 512), (64, 3, 2100), (72, 2, 512), (72, 1, 2100)])
def test_weights_of_few_queries_are_not_rounded_to_bf16(d, nq, nk):
    """Half of the keys weigh 2^-s and have the value 1, half weigh 1 and have what 8 bits hold of -2^-s, so that o nearly
    cancels and its own rounding is small: what is left is how far the weight 2^-s is off.  As a sum of two bf16 numbers it is off
    by 2^-15 of itself at most (a part that bf16 cuts off is below 2^-7, and half a step of that is 2^-8 of it), which
    moves o by half of it; bf16 alone misses some of these weights by 2^-9 and more."""
    rng = np.random.default_rng(43)
    for n16 in range(1, 16):
        c = Cache(1, d, [0, nk])
        k, v = torch.zeros(nk, 1, d), torch.zeros(nk, 1, d)
        low = torch.from_numpy(rng.permutation(nk) % 2 == 0)
        k[low, 0, 0] = -n16 / 16.0  # exact in 8 bits, and so are the scores
        v[:] = torch.where(low, 1.0, -float(O.kv8.round_e4m3(2.0 ** (-n16 / 16.0))))[:, None, None]
        c.store(k.bfloat16().cuda(), v.bfloat16().cuda())
        q = torch.zeros(nq, d, dtype=torch.bfloat16, device="cuda")
        q[:, 0] = 1.0
        ref, mag, _ = O.kv8.attention(f64(q).reshape(nq, 1, d), c.k, c.v, [0, nq], c.bounds)
        o = f64(attend(c, q, 1, [0, nq])).reshape(nq, 1, d)
        # o's rounding, the weights' (numerator), the exponential's and the sums' in fp32
        bound = 2.0 ** -8 * np.abs(ref) + (2.0 ** -15 + 2.02 * (2.0 ** -22 + (nk + 8) * 2.0 ** -24)) * mag
        assert (np.abs(o - ref) <= bound).all(), (n16, np.abs(o - ref).max(), bound.max())


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 72), ("f32", 64)])
def test_a_segment_packed_and_alone_is_the_same_up_to_rounding(dtype, d):
    """One query against 2100 keys, alone and beside 700 queries against 5000: another tile height and other chunks, so
    other sums and other roundings of the weights.  Each is held to the bound of its roundings, and what the segment's
    part of the cache holds is the same."""
    rng = np.random.default_rng(44)
    bf = dtype == "bf16"
    alone_plan, packed_plan = plan(2, [1], [2100], bf, d), plan(2, [700, 1], [5000, 2100], bf, d)
    assert alone_plan[1][0] != packed_plan[1][1] and (not bf or (alone_plan[0], packed_plan[0]) == (32, 128))
    packed = filled(rng, 2, d, [0, 2100, 7100], dtype)
    alone = Cache(2, d, [0, 2100])
    k, v = packed.load(dtype)
    alone.store(k[:2100].view(2100, 2, d), v[:2100].view(2100, 2, d), ld=2 * d)
    assert np.array_equal(alone.k, packed.k[:2100]) and np.array_equal(alone.v, packed.v[:2100])
    q = queries(rng, 701, 2, d, dtype)
    a = check_attention(alone, q[:1], 2, [0, 1])
    b = check_attention(packed, q, 2, [0, 1, 701])[:1]
    ref, mag, big = O.kv8.attention(f64(q[:1]).reshape(1, 2, d), alone.k, alone.v, [0, 1], alone.bounds)
    assert (np.abs(a - b) <= 2 * tolerance(dtype, ref, mag, big, 2100, d)).all()


@pytest.mark.parametrize("cleared", [True, False])
def test_a_new_sequence_in_an_old_ones_slice(cleared):
    """Cleared before, a block's first tokens are kept as if they were alone; otherwise the old rows behind them, which
    kv_len leaves out, still count for the scale."""
    rng = np.random.default_rng(45)
    c = Cache(2, 64, [0, 64])
    old = rows_of(rng, 64, 2, 64, "bf16") * 256
    c.store(old, old)
    if cleared:
        c.slice.zero_()
        c.k[:], c.v[:] = 0.0, 0.0
    new = torch.from_numpy(rng.standard_normal((5, 2, 64)).astype(np.float32)).bfloat16().cuda()
    c.store(new, new)
    c.check("f32")
    alone = O.kv8.quantise(f64(new), [0, 5])
    assert np.array_equal(c.k[:5], alone) == cleared
    check_attention(c, queries(rng, 1, 2, 64, "bf16"), 2, [0, 1], [5])


def test_the_tall_kernel_past_32_bit_offsets():
    """2^23 + 100 tokens of five heads (5.4 GB), 200 queries: the 128-row kernel.  All but a few rows are zero, so a
    zero key weighs 2^0; half of the queries score far past what a block's weights may sum to at the far end, where
    the block's scores are made again from its bytes."""
    n, heads = (1 << 23) + 100, 5
    rng = np.random.default_rng(46)
    assert plan(heads, [200], [n])[0] == 128
    size = B.sphinx_kv8_bytes(heads, 64, [0, n])
    assert size > 1 << 32
    cache = torch.zeros(size, dtype=torch.uint8, device="cuda")
    idx = np.array([0, 1 << 22, n - 170, n - 70, n - 2, n - 1], np.int32)
    k, v = (rng.standard_normal((6, heads, 64)) for _ in range(2))
    k, v = (torch.from_numpy(x.astype(np.float32)).bfloat16().cuda() for x in (k * 4, v * 1e6))
    B.sphinx_kv8_store(B.BF16, heads, 64, k, v, heads * 64, torch.from_numpy(idx).cuda(), 6, [0, n], cache)
    bounds = [0, 1, 2, 3, 4, 6]  # the last two share a block
    K, V = O.kv8.quantise(f64(k), bounds), O.kv8.quantise(f64(v), bounds)
    q = queries(rng, 200, heads, 64, "bf16") * 3
    q[::2] *= 8
    o = torch.empty(200, heads * 64, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(B.sphinx_kv8_attention_workspace_bytes(B.BF16, heads, heads, 64, [0, 200], [0, n]),
                     dtype=torch.uint8, device="cuda")
    B.sphinx_kv8_attention(B.BF16, heads, heads, 64, q, heads * 64, cache, [0, n], None, o, [0, 200], ws)
    qq = f64(q).reshape(200, heads, 64)
    s = np.einsum("qhd,thd->qht", qq, K)
    assert s.max() > 100.0
    top = np.maximum(s.max(2, keepdims=True), 0.0)
    w = np.exp2(s - top)
    den = w.sum(2) + (n - 6) * np.exp2(-top[..., 0])
    ref = np.einsum("qht,thd->qhd", w, V) / den[..., None]
    mag = np.einsum("qht,thd->qhd", w, np.abs(V)) / den[..., None]
    big = np.einsum("qhd,thd->qht", np.abs(qq), np.abs(K)).max(2)[..., None]
    # fp32 sums of 2^23 equal numbers, added in runs of at most 2^17 blocks, take 2^-7 of the sum, and weights 2^-8;
    # a score is off by 66 roundings of sum |q k|
    err = np.abs(f64(o).reshape(200, heads, 64) - ref)
    assert (err <= mag * (2.0 ** -6 + 2.02 * np.log(2.0) * 66 * 2.0 ** -24 * big) + 2.0 ** -8 * np.abs(ref)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_whole_slices_past_32_bit_offsets(dtype):
    """All rows of 2^24 + 70 tokens of two heads (4.3 GB) stored and read back: the first blocks, some in the middle and
    the last ones, the partial one among them, are what the oracle holds."""
    n, heads = (1 << 24) + 70, 2
    size = B.sphinx_kv8_bytes(heads, 64, [0, n])
    assert size > 1 << 32
    cache = torch.zeros(size, dtype=torch.uint8, device="cuda")
    code = B.BF16 if dtype == "bf16" else B.F32
    gen = torch.Generator(device="cuda").manual_seed(5)
    k, v = (torch.randn(n, heads * 64, generator=gen, device="cuda", dtype=TDT[dtype]) for _ in range(2))
    B.sphinx_kv8_store(code, heads, 64, k, v, heads * 64, None, n, [0, n], cache)
    spans = [(0, 128), (1 << 23, (1 << 23) + 128), ((1 << 24) - 128, n)]
    want = [[O.kv8.quantise(f64(x[a:b]).reshape(-1, heads, 64), [0, b - a]) for a, b in spans] for x in (k, v)]
    k.fill_(7.0)
    v.fill_(7.0)
    B.sphinx_kv8_load(code, heads, 64, cache, [0, n], None, n, k, v, heads * 64)
    for x, held in zip((k, v), want):
        for (a, b), h in zip(spans, held):
            assert np.array_equal(f64(x[a:b]).reshape(-1, heads, 64), h), (a, b)


@pytest.mark.parametrize("d,nq", [(64, 1), (64, 40), (64, 300), (72, 2), (72, 300)])
def test_weights_that_bf16_holds(d, nq):
    """Whole scores, so that every weight is a power of two, and values of both signs that nearly cancel, so that o's own
    rounding is small: what is left is fp32 sums.  A weight that is wrong by 2^-10 of itself would show."""
    rng = np.random.default_rng(47)
    nk = 1000
    c = Cache(2, d, [0, nk])
    k = torch.zeros(nk, 2, d)
    k[:, :, 0] = torch.from_numpy(-rng.integers(0, 8, (nk, 2)).astype(np.float32))
    v = torch.from_numpy(rng.choice([-1.0, 1.0], (nk, 2, d)).astype(np.float32))
    c.store(k.bfloat16().cuda(), v.bfloat16().cuda())
    q = torch.zeros(nq, 2 * d, dtype=torch.bfloat16, device="cuda")
    q[:, 0], q[:, d] = 1.0, 1.0
    ref, mag, _ = O.kv8.attention(f64(q).reshape(nq, 2, d), c.k, c.v, [0, nq], c.bounds)
    o = f64(attend(c, q, 2, [0, nq])).reshape(nq, 2, d)
    bound = 2.0 ** -8 * np.abs(ref) + 2.02 * (2.0 ** -22 + (nk + 8) * 2.0 ** -24) * mag
    assert (np.abs(o - ref) <= bound).all() and bound.mean() < 2.0 ** -10 / 2
