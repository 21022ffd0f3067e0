"""Thin ctypes binding of the 8-bit key-value cache (``include/moe_kv8.h``).

Argument marshalling and shape checks only: quantisation, attention and eviction run in the HIP library.  torch is
used for device memory and streams; every call goes to the current stream of the cache's device unless one is given.  On a
given stream the caller sees to it that the tensors are ready; they may be dropped as soon as the call returns, but for calls on
a ``torch.cuda.ExternalStream``, which need them until the stream is done.
"""
from __future__ import annotations

import ctypes as C

from . import binding as B

KV8_EXPORTS = ["moe_kv8_append", "moe_kv8_attend", "moe_kv8_attend_workspace_bytes", "moe_kv8_evict",
               "moe_kv8_evict_workspace_bytes", "moe_kv8_last_error"]


class MoeKv8Cache(C.Structure):
    _fields_ = [("n_seq", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("max_len", C.c_int32),
                ("block", C.c_int32), ("reserved", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p),
                ("k_scale", C.c_void_p), ("v_scale", C.c_void_p), ("position", C.c_void_p)]


class MoeKv8Step(C.Structure):
    _fields_ = [("n_rows", C.c_int32), ("max_new", C.c_int32), ("max_cached", C.c_int32), ("reserved", C.c_int32),
                ("row_offsets", C.c_void_p), ("cached", C.c_void_p), ("next_position", C.c_void_p)]


_lib = None


def load_library():
    """The shared library with the entry points of the 8-bit cache typed (fails loudly when missing)."""
    global _lib
    if _lib is None:
        lib = B.load_library()
        vp, i32, i64, P = C.c_void_p, C.c_int32, C.c_int64, C.POINTER
        cache, step = P(MoeKv8Cache), P(MoeKv8Step)
        lib.moe_kv8_append.argtypes = [vp, cache, step, vp, vp, i64, i64]
        lib.moe_kv8_attend_workspace_bytes.argtypes = [cache, step, i32, i32, P(i64)]
        lib.moe_kv8_attend.argtypes = [vp, cache, step, i32, vp, i64, i64, C.c_float, vp, i64, i64, vp, vp, vp, i64]
        lib.moe_kv8_evict_workspace_bytes.argtypes = [cache, i32, P(i64)]
        lib.moe_kv8_evict.argtypes = [vp, cache, vp, i32, i32, i32, vp, vp, vp, vp, vp, vp, i64]
        for name in KV8_EXPORTS:
            getattr(lib, name).restype = C.c_int
        lib.moe_kv8_last_error.restype = C.c_char_p
        _lib = lib
    return _lib


def _check(status: int):
    if status != B.MOE_OK:
        raise B.MoeError(status, load_library().moe_kv8_last_error().decode())


def _refuse(what: str):
    raise B.MoeError(B.MOE_ERR_INVALID_ARG, what)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _whole(t, name: str, dtype, shape):
    """`t` is a contiguous tensor of this type and shape."""
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        _refuse(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)}")
    return t


class Kv8Cache:
    """The cache of one layer: its tensors and the struct that describes them."""

    def __init__(self, k, v, k_scale, v_scale, block: int, position=None):
        import torch
        if k.dim() != 4:
            _refuse("k must have four dimensions [n_seq, n_kv_heads, max_len, head_dim]")
        n_seq, kv, max_len, hd = k.shape
        _whole(k, "k", torch.uint8, k.shape)
        _whole(v, "v", torch.uint8, k.shape)
        for t, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            _whole(t, name, torch.float32, (n_seq, kv, max_len // max(1, block)))
        if position is not None:
            _whole(position, "position", torch.int32, (n_seq, kv, max_len))
        self.k, self.v, self.k_scale, self.v_scale, self.position, self.block = k, v, k_scale, v_scale, position, block
        self.n_seq, self.n_kv_heads, self.max_len, self.head_dim = n_seq, kv, max_len, hd
        self.device, self.slots = k.device, k.shape[:3]
        self.tensors = (k, v, k_scale, v_scale, position)
        self.c = MoeKv8Cache(n_seq, kv, hd, max_len, block, 0, _ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale), _ptr(position))
        self.ref = C.byref(self.c)

    @classmethod
    def empty(cls, n_seq: int, n_kv_heads: int, head_dim: int, max_len: int, block: int = 64, device="cuda:0", positions=True):
        """A cache whose slots hold nothing yet."""
        import torch
        shape = (n_seq, n_kv_heads, max_len, head_dim)
        k, v = (torch.empty(shape, dtype=torch.uint8, device=device) for _ in "kv")
        ks, vs = (torch.empty(shape[:2] + (max_len // max(1, block),), device=device) for _ in "kv")
        return cls(k, v, ks, vs, block, torch.empty(shape[:3], dtype=torch.int32, device=device) if positions else None)


class Kv8Step:
    """The new tokens of one step.  `cached` and the other arrays are read when the kernels run, so they may be updated
    in place between steps (also between replays of a captured graph) within the bounds given here.  ``next_position`` may be
    left out for sequences that have never been evicted from."""

    def __init__(self, cached, n_rows: int, max_new: int, max_cached: int, row_offsets=None, next_position=None):
        import torch
        n_seq = cached.numel()
        _whole(cached, "cached", torch.int32, (n_seq,))
        if row_offsets is not None:
            _whole(row_offsets, "row_offsets", torch.int32, (n_seq + 1,))
        if next_position is not None:
            _whole(next_position, "next_position", torch.int32, (n_seq,))
        self.cached, self.row_offsets, self.next_position = cached, row_offsets, next_position
        self.n_seq, self.n_rows = n_seq, n_rows
        self.tensors = (cached, row_offsets, next_position)
        self.c = MoeKv8Step(n_rows, max_new, max_cached, 0, _ptr(row_offsets), _ptr(cached), _ptr(next_position))
        self.ref = C.byref(self.c)


def _stream(cache: Kv8Cache, stream):
    if stream is not None:
        return stream.cuda_stream
    import torch
    # the raw handle: a step has several calls of a few microseconds, and a Stream object costs two
    return torch._C._cuda_getCurrentRawStream(cache.device.index or 0)


def _rows(t, name: str, step: Kv8Step, cache: Kv8Cache, heads):
    """Strides of bf16 rows [n_rows or more, heads, head_dim], elements of a head side by side."""
    import torch
    shape, stride = t.shape, t.stride()
    if (t.dtype != torch.bfloat16 or len(shape) != 3 or shape[0] < step.n_rows or shape[2] != cache.head_dim
            or (heads is not None and shape[1] != heads) or stride[2] != 1):
        _refuse(f"{name} must be a bf16 tensor [{step.n_rows} or more, {'heads' if heads is None else heads}, {cache.head_dim}] "
                "with the last dimension contiguous")
    return stride


def _made_on(stream):
    """Where a workspace for work on `stream` is made: with that stream current, so that the allocator, which hands memory on
    in the order of the stream it was asked on, neither gives it away early nor gives out what another stream still uses."""
    import contextlib
    import torch
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _used(stream, *tensors):
    """Tensors of a call on `stream`: the caller may drop them behind the call, so the allocator is told who still uses them.
    Not of a stream that torch does not own: the allocator would ask it for an event when a tensor is freed, which may be after
    the stream's end."""
    import torch
    if isinstance(stream, torch.cuda.ExternalStream):
        return
    for t in tensors:
        if t is not None:
            t.record_stream(stream)


def _same_sequences(cache: Kv8Cache, step: Kv8Step):
    if step.n_seq != cache.n_seq:
        _refuse("the step is for another number of sequences")


def append(cache: Kv8Cache, step: Kv8Step, k_new, v_new, stream=None):
    """Quantises k_new and v_new [n_rows, n_kv_heads, head_dim] (bf16, the same strides) into the cache."""
    _same_sequences(cache, step)
    stride = _rows(k_new, "k_new", step, cache, cache.n_kv_heads)
    if _rows(v_new, "v_new", step, cache, cache.n_kv_heads) != stride:
        _refuse("k_new and v_new must have the same strides")
    _check(load_library().moe_kv8_append(_stream(cache, stream), cache.ref, step.ref, k_new.data_ptr(), v_new.data_ptr(),
                                         stride[0], stride[1]))
    if stream is not None:
        _used(stream, *cache.tensors, *step.tensors, k_new, v_new)


def attend_workspace_bytes(cache: Kv8Cache, step: Kv8Step, n_q_heads: int, with_weights: bool) -> int:
    n = C.c_int64(0)
    _check(load_library().moe_kv8_attend_workspace_bytes(cache.ref, step.ref, n_q_heads, int(with_weights), C.byref(n)))
    return int(n.value)


def attend_workspace(cache: Kv8Cache, step: Kv8Step, n_q_heads: int, with_weights: bool):
    import torch
    return torch.empty(attend_workspace_bytes(cache, step, n_q_heads, with_weights), dtype=torch.uint8, device=cache.device)


def attend(cache: Kv8Cache, step: Kv8Step, q, out, weight_in=None, weight_out=None, workspace=None, softmax_scale: float = 0.0,
           stream=None):
    """Attention of q [n_rows, n_q_heads, head_dim] over the cache into `out`, after the append of the same step."""
    import torch
    _same_sequences(cache, step)
    heads = q.shape[1] if q.dim() == 3 else None
    qs, os = _rows(q, "q", step, cache, None), _rows(out, "out", step, cache, heads)
    for t, name in ((weight_in, "weight_in"), (weight_out, "weight_out")):
        if t is not None:
            _whole(t, name, torch.float32, cache.slots)
    if workspace is None:
        with _made_on(stream):
            workspace = attend_workspace(cache, step, heads, weight_out is not None)
    _check(load_library().moe_kv8_attend(
        _stream(cache, stream), cache.ref, step.ref, heads, q.data_ptr(), qs[0], qs[1], softmax_scale,
        out.data_ptr(), os[0], os[1], _ptr(weight_in), _ptr(weight_out), workspace.data_ptr(), workspace.numel()))
    if stream is not None:
        _used(stream, *cache.tensors, *step.tensors, q, out, weight_in, weight_out, workspace)
    return out


def evict_workspace(cache: Kv8Cache, keep: int):
    import torch
    n = C.c_int64(0)
    _check(load_library().moe_kv8_evict_workspace_bytes(cache.ref, keep, C.byref(n)))
    return torch.empty(int(n.value), dtype=torch.uint8, device=cache.device)


def evict(cache: Kv8Cache, held, max_held: int, keep: int, recent: int, next_position, weight_in, weight_out=None,
          position_out=None, kept=None, workspace=None, stream=None):
    """Brings every sequence down to `keep` slots; weights go to `weight_out` (in place when None).  ``next_position`` may be
    None for sequences that have never been evicted from and began at position 0."""
    import torch
    if weight_out is None:
        weight_out = weight_in
    _whole(held, "held", torch.int32, (cache.n_seq,))
    if next_position is not None:
        _whole(next_position, "next_position", torch.int32, (cache.n_seq,))
    for t, name in ((weight_in, "weight_in"), (weight_out, "weight_out")):
        _whole(t, name, torch.float32, cache.slots)
    if position_out is not None:
        _whole(position_out, "position_out", torch.int32, cache.slots)
    if kept is not None:
        _whole(kept, "kept", torch.int32, cache.slots[:2] + (keep,))
    if workspace is None:
        with _made_on(stream):
            workspace = evict_workspace(cache, keep)
    _check(load_library().moe_kv8_evict(
        _stream(cache, stream), cache.ref, _ptr(held), max_held, keep, recent, _ptr(next_position), _ptr(weight_in),
        _ptr(weight_out), _ptr(position_out), _ptr(kept), workspace.data_ptr(), workspace.numel()))
    if stream is not None:
        _used(stream, *cache.tensors, held, next_position, weight_in, weight_out, position_out, kept, workspace)
