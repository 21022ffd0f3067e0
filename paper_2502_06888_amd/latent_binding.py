"""Thin ctypes binding of attention over a latent cache (``include/moe_latent.h``).

Argument marshalling and shape checks only.  Streams and the life of tensors are as in ``kv8_binding``, whose ``Kv8Step``
describes the new tokens here, too.
"""
from __future__ import annotations

import ctypes as C

from . import binding as B
from .kv8_binding import Kv8Step, MoeKv8Step, _made_on, _ptr, _refuse, _same_sequences, _stream, _used, _whole
from .rope_binding import MoeRopeConfig, Rope

LATENT_EXPORTS = ["moe_latent_append", "moe_latent_attend", "moe_latent_attend_workspace_bytes", "moe_latent_last_error"]
FORMS = {"auto": 0, "absorbed": 1, "expanded": 2}


class MoeLatentCache(C.Structure):
    _fields_ = [("n_seq", C.c_int32), ("latent_dim", C.c_int32), ("rope_dim", C.c_int32), ("max_len", C.c_int32),
                ("prefix_len", C.c_int32), ("reserved", C.c_int32), ("rows", C.c_void_p), ("prefix", C.c_void_p)]


class MoeLatentHeads(C.Structure):
    _fields_ = [("n_heads", C.c_int32), ("nope_dim", C.c_int32), ("v_dim", C.c_int32), ("reserved", C.c_int32),
                ("w_k", C.c_void_p), ("w_v", C.c_void_p), ("w_k_head", C.c_int64), ("w_v_head", C.c_int64)]


_lib = None


def load_library():
    """The shared library with the entry points of the latent cache typed (fails loudly when missing)."""
    global _lib
    if _lib is None:
        lib = B.load_library()
        vp, i32, i64, P = C.c_void_p, C.c_int32, C.c_int64, C.POINTER
        cache, step, heads = P(MoeLatentCache), P(MoeKv8Step), P(MoeLatentHeads)
        lib.moe_latent_append.argtypes = [vp, cache, step, vp, i64, vp, C.c_float, P(MoeRopeConfig)]
        lib.moe_latent_attend_workspace_bytes.argtypes = [cache, step, heads, i32, P(i64)]
        lib.moe_latent_attend.argtypes = [vp, cache, step, heads, vp, i64, i64, C.c_float, i32, vp, i64, i64, vp, i64]
        for name in LATENT_EXPORTS:
            getattr(lib, name).restype = C.c_int
        lib.moe_latent_last_error.restype = C.c_char_p
        _lib = lib
    return _lib


def _check(status: int):
    if status != B.MOE_OK:
        raise B.MoeError(status, load_library().moe_latent_last_error().decode())


class LatentCache:
    """The cache of one layer: rows [n_seq, max_len, latent + rope_dim] (bf16) and, where the sequences share one, the prefix
    [prefix_len, latent + rope_dim] they all see before their own rows."""

    def __init__(self, rows, rope_dim: int, prefix=None):
        import torch
        if rows.dim() != 3:
            _refuse("rows must have three dimensions [n_seq, max_len, latent + rope_dim]")
        n_seq, max_len, width = rows.shape
        _whole(rows, "rows", torch.bfloat16, rows.shape)
        if prefix is not None:
            _whole(prefix, "prefix", torch.bfloat16, (prefix.shape[0], width))
        self.rows, self.prefix, self.rope_dim = rows, prefix, rope_dim
        self.n_seq, self.max_len, self.latent_dim = n_seq, max_len, width - rope_dim
        self.device, self.tensors = rows.device, (rows, prefix)
        self.c = MoeLatentCache(n_seq, width - rope_dim, rope_dim, max_len, 0 if prefix is None else prefix.shape[0], 0, _ptr(rows),
                                _ptr(prefix))
        self.ref = C.byref(self.c)

    @classmethod
    def empty(cls, n_seq: int, max_len: int, latent_dim: int = 512, rope_dim: int = 64, prefix=None, device="cuda:0"):
        """A cache whose slots hold nothing yet."""
        import torch
        return cls(torch.empty((n_seq, max_len, latent_dim + rope_dim), dtype=torch.bfloat16, device=device), rope_dim, prefix)


def _weights(w, name: str, latent: int):
    """Heads of [rows, latent], rows one behind the other; heads may lie apart (parts of one matrix)."""
    import torch
    if w.dtype != torch.bfloat16 or w.dim() != 3 or w.shape[2] != latent or w.stride(2) != 1 or w.stride(1) != latent:
        _refuse(f"{name} must be a bf16 tensor [n_heads, rows, latent] whose heads are contiguous")
    if w.shape[0] > 1 and w.stride(0) == 0:
        _refuse(f"the heads of {name} must be there one by one")
    return w.stride(0) if w.shape[0] > 1 else 0


class LatentHeads:
    """The matrices of the heads: w_k [n_heads, nope_dim, latent], w_v [n_heads, v_dim, latent] (bf16)."""

    def __init__(self, w_k, w_v):
        if w_k.dim() != 3 or w_v.dim() != 3 or w_k.shape[0] != w_v.shape[0] or w_k.shape[2] != w_v.shape[2]:
            _refuse("w_k and w_v must be [n_heads, nope_dim, latent] and [n_heads, v_dim, latent]")
        self.w_k, self.w_v = w_k, w_v
        self.n, self.nope_dim, self.latent_dim = w_k.shape
        self.v_dim, self.tensors = w_v.shape[1], (w_k, w_v)
        self.c = MoeLatentHeads(self.n, self.nope_dim, self.v_dim, 0, _ptr(w_k), _ptr(w_v), _weights(w_k, "w_k", self.latent_dim),
                                _weights(w_v, "w_v", self.latent_dim))
        self.ref = C.byref(self.c)


def append(cache: LatentCache, step: Kv8Step, x, norm=None, eps: float = 1e-6, rope: Rope = None, stream=None):
    """Writes the rows x [n_rows, latent + rope_dim] (bf16) of the new tokens into the cache: latents normalised and times `norm`
    (bf16 [latent]) where it is given, the other part turned by the tokens' positions where `rope` is."""
    import torch
    _same_sequences(cache, step)
    width = cache.latent_dim + cache.rope_dim
    if x.dtype != torch.bfloat16 or x.dim() != 2 or x.shape[0] < step.n_rows or x.shape[1] != width or x.stride(1) != 1:
        _refuse(f"x must be a bf16 tensor [{step.n_rows} or more, {width}] with the last dimension contiguous")
    if norm is not None:
        _whole(norm, "norm", torch.bfloat16, (cache.latent_dim,))
    _check(load_library().moe_latent_append(_stream(cache, stream), cache.ref, step.ref, x.data_ptr(), x.stride(0), _ptr(norm), eps,
                                            None if rope is None else rope.ref))
    if stream is not None:
        _used(stream, *cache.tensors, *step.tensors, x, norm)


def attend_workspace_bytes(cache: LatentCache, step: Kv8Step, heads: LatentHeads, form: str = "auto") -> int:
    if form not in FORMS:
        _refuse(f"form must be one of {', '.join(FORMS)}")
    n = C.c_int64(0)
    _check(load_library().moe_latent_attend_workspace_bytes(cache.ref, step.ref, heads.ref, FORMS[form], C.byref(n)))
    return int(n.value)


def attend_workspace(cache: LatentCache, step: Kv8Step, heads: LatentHeads, form: str = "auto"):
    import torch
    return torch.empty(attend_workspace_bytes(cache, step, heads, form), dtype=torch.uint8, device=cache.device)


def _rows(t, name: str, n_rows: int, heads: int, width: int):
    import torch
    if t.dtype != torch.bfloat16 or t.dim() != 3 or t.shape[0] < n_rows or t.shape[1:] != (heads, width) or t.stride(2) != 1:
        _refuse(f"{name} must be a bf16 tensor [{n_rows} or more, {heads}, {width}] with the last dimension contiguous")
    return t.stride()


def attend(cache: LatentCache, step: Kv8Step, heads: LatentHeads, q, out, softmax_scale: float = 0.0, form: str = "auto",
           workspace=None, stream=None):
    """Attention of q [n_rows, n_heads, nope_dim + rope_dim] (its last rope_dim elements turned) over the cache into `out`
    [n_rows, n_heads, v_dim], after the append of the same step."""
    _same_sequences(cache, step)
    if heads.latent_dim != cache.latent_dim:
        _refuse("the heads are for another latent dimension")
    if form not in FORMS:
        _refuse(f"form must be one of {', '.join(FORMS)}")
    qs = _rows(q, "q", step.n_rows, heads.n, heads.nope_dim + cache.rope_dim)
    os = _rows(out, "out", step.n_rows, heads.n, heads.v_dim)
    if workspace is None:
        with _made_on(stream):
            workspace = attend_workspace(cache, step, heads, form)
    _check(load_library().moe_latent_attend(
        _stream(cache, stream), cache.ref, step.ref, heads.ref, q.data_ptr(), qs[0], qs[1], softmax_scale, FORMS[form], out.data_ptr(),
        os[0], os[1], workspace.data_ptr(), workspace.numel()))
    if stream is not None:
        _used(stream, *cache.tensors, *step.tensors, *heads.tensors, q, out, workspace)
    return out
