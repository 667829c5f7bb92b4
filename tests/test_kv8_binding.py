"""Tensors and host integers that the calls of the 8-bit cache refuse before anything is launched (no GPU needed)."""
import os

import numpy as np
import pytest

import workloads as W

torch = pytest.importorskip("torch")
S = pytest.importorskip("paper_2511_18672_amd")
B = S.binding

BF, F = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def built():
    if not os.path.exists(B.LIB_PATH):
        pytest.skip("libsphinx.so not built")


def rows(n, width, dtype=BF):
    return torch.zeros(n, width, dtype=dtype)


def store(dtype=B.BF16, k=None, v=None, ld=128, n=8, cu=(0, 64), cache=None):
    k, v = rows(8, 128) if k is None else k, rows(8, 128) if v is None else v
    B.sphinx_kv8_store(dtype, 2, 64, k, v, ld, None, n, cu, torch.zeros(40000, dtype=torch.uint8) if cache is None else cache)


def load(dtype=B.BF16, k=None, v=None, ld=128, n=8, cu=(0, 64), cache=None):
    k, v = rows(8, 128) if k is None else k, rows(8, 128) if v is None else v
    B.sphinx_kv8_load(dtype, 2, 64, torch.zeros(40000, dtype=torch.uint8) if cache is None else cache, cu, None, n, k, v, ld)


def attend(dtype=B.BF16, q=None, ldq=256, o=None, cu_q=(0, 5), cu_kv=(0, 64), kv_len=None, cache=None, ws=None):
    q, o = rows(5, 256) if q is None else q, rows(5, 256) if o is None else o
    some = torch.zeros(1 << 20, dtype=torch.uint8)
    B.sphinx_kv8_attention(dtype, 4, 2, 64, q, ldq, some if cache is None else cache, cu_kv, kv_len, o, cu_q,
                           some if ws is None else ws)


@pytest.mark.parametrize("call", [store, load])
def test_rows_of_another_type_or_too_few_are_refused(call):
    for name in ("k", "v"):
        for bad in (rows(8, 128, F), rows(8, 128, torch.float16), rows(8, 64), rows(7, 128), rows(1, 128).expand(8, 128)):
            with pytest.raises(ValueError, match=name + " "):
                call(**{name: bad})
    with pytest.raises(ValueError, match="another type"):
        call(dtype=B.F32)
    with pytest.raises(ValueError, match="elements"):
        call(ld=256)


def test_queries_and_outputs_of_another_type_or_too_few_are_refused():
    for bad in (rows(5, 256, F), rows(5, 256, torch.float16), rows(4, 256), rows(5, 128)):
        with pytest.raises(ValueError, match="q "):
            attend(q=bad)
        with pytest.raises(ValueError, match="o "):
            attend(o=bad)
    with pytest.raises(ValueError, match="q "):
        attend(ldq=512)
    with pytest.raises(ValueError, match="another type"):
        attend(dtype=B.F32)


def test_rows_that_their_memory_holds_are_taken():
    wide = torch.zeros(8, 384, dtype=BF)
    for t, n, ld in ((rows(8, 128), 8, 128), (rows(8, 128), 3, 128), (wide[:, 128:256], 8, 384), (wide[:, 256:], 8, 384),
                     (wide[:, 256:].unflatten(1, (2, 64)), 8, 384), (wide[0, 256:], 8, 384), (wide.view(-1)[256:], 8, 384),
                     (rows(0, 128), 0, 128), (torch.zeros(8 * 128, dtype=BF), 8, 128)):
        B._check_rows("k", t, B.BF16, n, ld, 128)
    B._check_rows("k", torch.zeros(7 * 256 + 128, dtype=BF), B.BF16, 8, 256, 128)
    with pytest.raises(ValueError):  # the last row ends one element behind the memory
        B._check_rows("k", torch.zeros(7 * 256 + 127, dtype=BF), B.BF16, 8, 256, 128)


@pytest.mark.parametrize("call", [store, load, attend])
def test_slices_that_are_not_bytes_in_a_row_are_refused(call):
    some = torch.zeros(1 << 21, dtype=torch.uint8)
    for bad in (some[::2], torch.zeros(1, dtype=torch.uint8).expand(1 << 20)):
        with pytest.raises(ValueError, match="in a row"):
            call(cache=bad)
        if call is attend:
            with pytest.raises(ValueError, match="in a row"):
                call(ws=bad)


def test_token_bounds_that_are_not_32_bit_integers_are_refused():
    big = (1 << 32) + 64  # as an int32 it would be 64
    for bad in (np.array([0, big]), [0, big], [0, -big], np.array([0, 64], np.uint64) + np.uint64(1 << 32), [0.0, 64.0],
                np.array([[0, 64]]), np.array([[0, 64]], np.int32)):
        for call in (lambda cu: B.sphinx_kv8_bytes(2, 64, cu), lambda cu: store(cu=cu), lambda cu: load(cu=cu),
                     lambda cu: attend(cu_kv=cu), lambda cu: attend(cu_q=cu), lambda cu: attend(kv_len=cu),
                     lambda cu: B.sphinx_kv8_attention_workspace_bytes(B.BF16, 4, 2, 64, [0, 5], cu)):
            with pytest.raises(ValueError):
                call(bad)
    for good in ([0, 64], np.array([0, 64]), np.array([0, 64], np.uint8), np.array([0, 9, 64, 9], np.int32)[::2], torch.tensor([0, 64])):
        assert B.sphinx_kv8_bytes(2, 64, good) == 2 * 2 * 64 * 64 + 256


def test_a_cache_of_too_few_bytes_for_its_requests_is_refused():
    reqs = S.make_requests([W.Request(2, 8, 8)])
    desc = S.model_desc(W.SMALL_MODEL, 256)
    need = S.sphinx_kv8_cache_bytes(desc, reqs)
    x = torch.zeros(16 * 32)
    with pytest.raises(ValueError, match="bytes"):
        S.sphinx_refine_step_kv8(desc, reqs, x, 5, np.array([0, 5]), x, x, x, x, torch.zeros(need - 1, dtype=torch.uint8),
                                 torch.zeros(256, dtype=torch.uint8), 0)


def test_streams_of_another_device_are_refused(monkeypatch):
    class Stream:
        def __init__(self, device_index):
            self.device_index, self.cuda_stream = device_index, 77

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises(ValueError, match="stream of cuda:0"):
        B._here(Stream(0))
    assert B._here(Stream(1)) == 77 and B._here(5) == 5
