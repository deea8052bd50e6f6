"""ctypes binding of libmi355seq.so: the C ABI of include/mi355seq.h, same names.

Argument marshalling only; device pointers are plain integers and streams are
``hipStream_t`` handles.  There is no fallback: if the library is missing,
importing this module fails.
"""
from __future__ import annotations

import ctypes
import functools
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmi355seq.so")

SEQ_FP32 = 0
SEQ_FP16 = 1
SEQ_BF16 = 2
SEQ_OK = 0
SEQ_EINVAL = -1
SEQ_EUNSUPPORTED = -2
SEQ_EALIGN = -4
SEQ_EHIP = -5
SEQ_SCAN_CHUNK = 16

# every symbol include/mi355seq.h declares
EXPORTS = ("seq_scan_forward", "seq_scan_backward", "seq_scan_saved_bytes", "seq_scan_workspace_bytes",
           "seq_norm_forward", "seq_norm_backward", "seq_norm_workspace_bytes", "seq_strerror")

if not os.path.exists(LIB_PATH):
    raise ImportError(
        f"{LIB_PATH} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'` "
        "(there is no CPU fallback)")

lib = ctypes.CDLL(LIB_PATH)
_i64, _vp, _int, _float = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_float
lib.seq_scan_forward.argtypes = [_i64, _i64, _i64, _int] + [_vp] * 12
lib.seq_scan_forward.restype = _int
lib.seq_scan_backward.argtypes = [_i64, _i64, _i64, _int] + [_vp] * 16
lib.seq_scan_backward.restype = _int
lib.seq_scan_saved_bytes.argtypes = [_i64, _i64, _i64]
lib.seq_scan_saved_bytes.restype = ctypes.c_size_t
lib.seq_scan_workspace_bytes.argtypes = [_i64, _i64, _i64, _int, _int]
lib.seq_scan_workspace_bytes.restype = ctypes.c_size_t
lib.seq_norm_forward.argtypes = [_i64, _i64, _int] + [_vp] * 7 + [_float] + [_vp] * 4
lib.seq_norm_forward.restype = _int
lib.seq_norm_backward.argtypes = [_i64, _i64, _int] + [_vp] * 9 + [_float] + [_vp] * 9
lib.seq_norm_backward.restype = _int
lib.seq_norm_workspace_bytes.argtypes = [_i64, _i64, _int]
lib.seq_norm_workspace_bytes.restype = ctypes.c_size_t
lib.seq_strerror.argtypes = [_int]
lib.seq_strerror.restype = ctypes.c_char_p


class SeqError(RuntimeError):
    def __init__(self, code: int, what: str):
        super().__init__(f"{what}: {seq_strerror(code)} ({code})")
        self.code = code


def check(code: int, what: str) -> None:
    if code != SEQ_OK:
        raise SeqError(code, what)


def seq_strerror(code: int) -> str:
    return lib.seq_strerror(code).decode()


_array_of = functools.lru_cache(maxsize=None)(lambda n: ctypes.c_int64 * n)


def int64s(values):
    """A host array of 64-bit strides."""
    return _array_of(len(values))(*values)
