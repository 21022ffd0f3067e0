"""Thin ctypes binding of rotary positions (``include/moe_rope.h``).

Argument marshalling and shape checks only.  Calls go to the current stream of the rows' device unless one is given, as in
``kv8_binding``.
"""
from __future__ import annotations

import ctypes as C

from . import binding as B
from .kv8_binding import _refuse, _used, _whole

ROPE_EXPORTS = ["moe_rope_last_error", "moe_rope_rotate"]


class MoeRopeConfig(C.Structure):
    _fields_ = [("rot_dim", C.c_int32), ("first", C.c_int32), ("interleaved", C.c_int32), ("original_len", C.c_int32),
                ("theta", C.c_double), ("factor", C.c_double), ("low_turns", C.c_double), ("high_turns", C.c_double),
                ("magnitude", C.c_double)]


class MoeRopeRows(C.Structure):
    _fields_ = [("in_", C.c_void_p), ("out", C.c_void_p), ("n_heads", C.c_int32), ("reserved", C.c_int32),
                ("in_row", C.c_int64), ("in_head", C.c_int64), ("out_row", C.c_int64), ("out_head", C.c_int64)]


_lib = None


def load_library():
    """The shared library with the entry points of rotary positions typed (fails loudly when missing)."""
    global _lib
    if _lib is None:
        lib = B.load_library()
        vp, i32, P = C.c_void_p, C.c_int32, C.POINTER
        lib.moe_rope_rotate.argtypes = [vp, P(MoeRopeConfig), i32, i32, i32, vp, P(MoeRopeRows), P(MoeRopeRows)]
        lib.moe_rope_rotate.restype = C.c_int
        lib.moe_rope_last_error.restype = C.c_char_p
        _lib = lib
    return _lib


class Rope:
    """What turns and how fast: `rot_dim` elements from `first` on of every head, frequencies of base `theta`, divided by `factor`, or
    by parts of it where `original_len` is given."""

    def __init__(self, rot_dim: int, theta: float = 10000.0, first: int = 0, interleaved: bool = False, factor: float = 1.0,
                 original_len: int = 0, low_turns: float = 1.0, high_turns: float = 32.0, magnitude: float = 1.0):
        self.c = MoeRopeConfig(rot_dim, first, int(interleaved), original_len, theta, factor, low_turns, high_turns, magnitude)
        self.ref = C.byref(self.c)


def _rows(x, out, name: str, like, dtypes):
    """The struct of rows [n_rows, heads, head_dim]; `out` None: in place."""
    if out is None:
        out = x
    for t, n in ((x, name), (out, name + "_out")):
        if t.dim() != 3 or t.dtype != like.dtype or t.dtype not in dtypes or t.shape != (like.shape[0], x.shape[1], like.shape[2]) or t.stride(2) != 1:
            _refuse(f"{n} must be a bf16 or float32 tensor [n_rows, heads, head_dim] with the last dimension contiguous, all rows of one "
                    "type, n_rows and head_dim")
    a, b = x.stride(), out.stride()
    return MoeRopeRows(x.data_ptr(), out.data_ptr(), x.shape[1], 0, a[0], a[1], b[0], b[1])


def rotate(rope: Rope, positions, q, q_out=None, k=None, k_out=None, stream=None):
    """Turns q and k [n_rows, heads, head_dim] by `positions` (int32 [n_rows]), in place where no output is given."""
    import torch
    dtypes = (torch.bfloat16, torch.float32)
    rq = _rows(q, q_out, "q", q, dtypes)
    rk = None
    if k is not None:
        rk = _rows(k, k_out, "k", q, dtypes)
    elif k_out is not None:
        _refuse("k_out without k")
    _whole(positions, "positions", torch.int32, (q.shape[0],))
    lib = load_library()
    raw = torch._C._cuda_getCurrentRawStream(q.device.index or 0) if stream is None else stream.cuda_stream
    status = lib.moe_rope_rotate(raw, rope.ref, B.MOE_F32 if q.dtype == torch.float32 else B.MOE_BF16, q.shape[0], q.shape[2],
                                 positions.data_ptr(), C.byref(rq), None if rk is None else C.byref(rk))
    if status != B.MOE_OK:
        raise B.MoeError(status, lib.moe_rope_last_error().decode())
    if stream is not None:
        _used(stream, positions, q, q_out, k, k_out)
