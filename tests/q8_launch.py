"""launch_q8_matmul of the library itself (csrc/q8.hpp): the products inside a refinement step, which have no entry
point of their own, for tests that compare them alone."""
import ctypes
from ctypes import POINTER, c_bool, c_float, c_int32, c_int64, c_void_p

BF16, F32, GATED, BYTES = range(4)  # Q8Kind
STORE, GELU, ADD = range(3)         # Q8_EPI_*
SYMBOL = "_ZN6sphinx16launch_q8_matmulENS_6Q8KindEiiiRKNS_5Q8MatES3_RKNS_5Q8EpiEPfP12ihipStream_t"


class Q8Mat(ctypes.Structure):
    _fields_ = [("q", c_void_p), ("s", c_void_p)]


class Q8Epi(ctypes.Structure):
    _fields_ = [("epi", c_int32), ("bias", c_void_p), ("bias_bf16", c_bool), ("out", c_void_p), ("ldo", c_int64),
                ("scales", c_void_p), ("gate", c_void_p), ("ldg", c_int64), ("row_of", c_void_p), ("qcols", c_int32),
                ("qscale", c_float)]


def layout_checks():
    """C++ that compiles only if both structures are laid out as here."""
    lines = ['#include <cstddef>', '#include "q8.hpp"', "using namespace sphinx;"]
    for t in (Q8Mat, Q8Epi):
        lines.append(f'static_assert(sizeof({t.__name__}) == {ctypes.sizeof(t)}, "size");')
        lines += [f'static_assert(offsetof({t.__name__}, {n}) == {getattr(t, n).offset}, "{n}");' for n, _ in t._fields_]
    lines += [f'static_assert({n} == {v}, "{n}");' for n, v in
              (("kQ8Bf16", BF16), ("kQ8F32", F32), ("kQ8Gated", GATED), ("kQ8Bytes", BYTES), ("Q8_EPI_STORE", STORE),
               ("Q8_EPI_GELU", GELU), ("Q8_EPI_ADD", ADD))]
    return "\n".join(lines) + "\n"


def launch(lib, kind, M, N, K, a, b, ws=None, stream=None, **epilogue):
    """Returns the hipError_t.  a, b: (bytes, scales); pointers of the epilogue by name, as tensors."""
    f = getattr(lib, SYMBOL)
    f.restype = c_int32
    f.argtypes = [c_int32, c_int32, c_int32, c_int32, POINTER(Q8Mat), POINTER(Q8Mat), POINTER(Q8Epi), c_void_p, c_void_p]
    p = lambda t: t.data_ptr() if hasattr(t, "data_ptr") else t  # noqa: E731
    e = Q8Epi(**{k: p(v) for k, v in epilogue.items()})
    return f(kind, M, N, K, Q8Mat(*map(p, a)), Q8Mat(*map(p, b)), e, p(ws), stream)
