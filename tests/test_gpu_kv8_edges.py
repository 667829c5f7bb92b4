"""The 8-bit key/value cache through the C ABI: sums that overflow late in a block, weights that bf16 misses, segments
packed and alone."""
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
