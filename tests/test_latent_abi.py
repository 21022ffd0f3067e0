"""Rotary positions and the latent cache without a GPU: exported symbols, struct sizes, sizing, refusals that the host decides."""
import ctypes as C
import math
import os
import re

import pytest
import torch

from oracle import latent_ref as R
from paper_2502_06888_amd import binding as B
from paper_2502_06888_amd import kv8_binding as Q
from paper_2502_06888_amd import latent_binding as L
from paper_2502_06888_amd import rope_binding as P

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def ints(*v):
    return torch.tensor(v, dtype=torch.int32)


def parts(n_seq=2, max_len=128, latent=512, rope=64, heads=8, nope=128, value=128, prefix=0):
    cache = L.LatentCache.empty(n_seq, max_len, latent, rope, device="cpu",
                                prefix=torch.zeros((prefix, latent + rope), dtype=torch.bfloat16) if prefix else None)
    return cache, L.LatentHeads(*(torch.zeros((heads, n, latent), dtype=torch.bfloat16) for n in (nope, value)))


def exported(header, prefix):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", header)).read(), flags=re.S)
    return sorted(set(re.findall(r"\b(" + prefix + r"_[a-z0-9_]+)\s*\(", text)))


def test_library_exports_every_symbol():
    assert exported("moe_rope.h", "moe_rope") == sorted(P.ROPE_EXPORTS)
    assert exported("moe_latent.h", "moe_latent") == sorted(L.LATENT_EXPORTS)
    for lib, names in ((P.load_library(), P.ROPE_EXPORTS), (L.load_library(), L.LATENT_EXPORTS)):
        for n in names:
            assert hasattr(lib, n)
    assert C.sizeof(P.MoeRopeConfig) == 4 * 4 + 5 * 8 and C.sizeof(P.MoeRopeRows) == 2 * 8 + 2 * 4 + 4 * 8
    assert C.sizeof(L.MoeLatentCache) == 6 * 4 + 2 * 8 and C.sizeof(L.MoeLatentHeads) == 4 * 4 + 4 * 8


@pytest.mark.parametrize("field,value,status", [
    ("n_seq", 0, B.MOE_ERR_SHAPE), ("n_seq", 65537, B.MOE_ERR_SHAPE), ("latent_dim", 64, B.MOE_ERR_SHAPE), ("latent_dim", 384, B.MOE_ERR_SHAPE),
    ("rope_dim", 16, B.MOE_ERR_SHAPE), ("rope_dim", 128, B.MOE_ERR_SHAPE), ("max_len", 0, B.MOE_ERR_SHAPE),
    ("max_len", (1 << 20) + 1, B.MOE_ERR_SHAPE), ("prefix_len", -1, B.MOE_ERR_SHAPE), ("prefix_len", (1 << 20) + 1, B.MOE_ERR_SHAPE),
    ("reserved", 1, B.MOE_ERR_INVALID_ARG),
])
def test_sizes_of_the_cache_are_checked(field, value, status):
    c, h = parts()
    setattr(c.c, field, value)
    with pytest.raises(B.MoeError) as e:
        L.attend_workspace_bytes(c, Q.Kv8Step(ints(3, 4), 2, 1, 4), h)
    assert e.value.status == status and e.value.message


@pytest.mark.parametrize("field,value,status", [
    ("n_heads", 0, B.MOE_ERR_SHAPE), ("n_heads", 257, B.MOE_ERR_SHAPE), ("nope_dim", 96, B.MOE_ERR_SHAPE), ("nope_dim", 256, B.MOE_ERR_SHAPE),
    ("v_dim", 16, B.MOE_ERR_SHAPE), ("reserved", 3, B.MOE_ERR_INVALID_ARG), ("w_k_head", -8, B.MOE_ERR_INVALID_ARG),
    ("w_v_head", 4, B.MOE_ERR_INVALID_ARG),
])
def test_sizes_of_the_heads_are_checked(field, value, status):
    c, h = parts()
    setattr(h.c, field, value)
    with pytest.raises(B.MoeError) as e:
        L.attend_workspace_bytes(c, Q.Kv8Step(ints(3, 4), 2, 1, 4), h)
    assert e.value.status == status and e.value.message


@pytest.mark.parametrize("rows,new,cached,offsets,status", [
    (-1, 1, 4, True, B.MOE_ERR_SHAPE), ((1 << 20) + 1, 1, 4, True, B.MOE_ERR_SHAPE), (2, -1, 4, True, B.MOE_ERR_INVALID_ARG),
    (2, 1, -1, True, B.MOE_ERR_INVALID_ARG), (2, 1, 129, True, B.MOE_ERR_INVALID_ARG), (2, 129, 4, True, B.MOE_ERR_INVALID_ARG),
    (3, 1, 4, False, B.MOE_ERR_INVALID_ARG), (2, 0, 4, True, B.MOE_ERR_INVALID_ARG), (0, 1, 4, True, B.MOE_ERR_INVALID_ARG),
])
def test_bounds_of_a_step_are_checked(rows, new, cached, offsets, status):
    c, h = parts()
    s = Q.Kv8Step(ints(3, 4), rows, new, cached, row_offsets=ints(0, 1, 2) if offsets else None)
    with pytest.raises(B.MoeError) as e:
        L.attend_workspace_bytes(c, s, h)
    assert e.value.status == status and e.value.message
    lib = L.load_library()
    assert lib.moe_latent_append(None, c.ref, s.ref, None, 576, None, 0.0, None) == status


@pytest.mark.parametrize("dims", [(512, 64, 128, 128), (256, 32, 64, 64), (128, 32, 32, 128)])
@pytest.mark.parametrize("seqs,heads,prefix", [(1, 1, 0), (2, 20, 700), (64, 128, 0), (64, 5, 1 << 20)])
def test_workspace_is_found_for_every_bound(seqs, heads, prefix, dims):
    c, h = parts(n_seq=1, max_len=1, latent=dims[0], rope=dims[1], heads=heads, nope=dims[2], value=dims[3])
    c.n_seq, c.c.n_seq, c.c.max_len, c.c.prefix_len = seqs, seqs, 1 << 16, prefix
    for new in (0, 1, 4, 17, 1000, 65536):
        for cached in (0, 1, 63, 2000, 65536):
            for rows in sorted({min(new, 1), new, min(seqs * new, 1 << 20)}):
                s = Q.Kv8Step(ints(*[0] * seqs), rows, new, cached, row_offsets=ints(*[0] * (seqs + 1)))
                for form in L.FORMS:
                    try:
                        assert (L.attend_workspace_bytes(c, s, h, form) > 0) == (rows > 0)
                    except B.MoeError as e:
                        assert rows >= 1000 and "workgroups" in e.message


def test_more_workgroups_than_a_launch_has_are_refused():
    c, h = parts(max_len=1, heads=256)
    c.c.n_seq, c.c.max_len = 65536, 1 << 20
    with pytest.raises(B.MoeError) as e:
        L.attend_workspace_bytes(c, Q.Kv8Step(ints(0), 1 << 20, 1 << 20, 0, row_offsets=ints(0, 1)), h, "absorbed")
    assert e.value.status == B.MOE_ERR_SHAPE and "workgroups" in e.value.message


def test_null_arguments_host_tensors_forms_and_scales_are_refused():
    lib, (c, h), s = L.load_library(), parts(), Q.Kv8Step(ints(3, 4), 2, 1, 4)
    n, bad = C.c_int64(0), B.MOE_ERR_INVALID_ARG
    assert lib.moe_latent_attend_workspace_bytes(None, s.ref, h.ref, 0, C.byref(n)) == bad
    assert lib.moe_latent_attend_workspace_bytes(c.ref, None, h.ref, 0, C.byref(n)) == bad
    assert lib.moe_latent_attend_workspace_bytes(c.ref, s.ref, None, 0, C.byref(n)) == bad
    assert lib.moe_latent_attend_workspace_bytes(c.ref, s.ref, h.ref, 0, None) == bad
    for form in (-1, 3):
        assert lib.moe_latent_attend_workspace_bytes(c.ref, s.ref, h.ref, form, C.byref(n)) == bad
    for scale in (-1.0, math.inf, math.nan, 3.0e38):
        assert lib.moe_latent_attend(None, c.ref, s.ref, h.ref, None, 0, 0, scale, 0, None, 0, 0, None, 0) == bad
        assert b"softmax_scale" in lib.moe_latent_last_error()
    assert lib.moe_latent_attend(None, c.ref, s.ref, h.ref, None, 0, 0, 0.0, 0, None, 0, 0, None, 0) == bad
    assert b"cache.rows is not device memory" in lib.moe_latent_last_error()
    assert lib.moe_latent_append(None, c.ref, s.ref, None, 576, None, 0.0, None) == bad
    assert b"cache.rows is not device memory" in lib.moe_latent_last_error()
    for eps in (-1.0, math.nan, math.inf):
        assert lib.moe_latent_append(None, c.ref, s.ref, None, 576, 16, eps, None) == bad
        assert b"eps" in lib.moe_latent_last_error()
    for rope in (P.Rope(128), P.Rope(64, first=2), P.Rope(32, first=40)):
        assert lib.moe_latent_append(None, c.ref, s.ref, None, 576, None, 0.0, rope.ref) == B.MOE_ERR_SHAPE


def test_shapes_the_binding_refuses():
    c, h = parts()
    s = Q.Kv8Step(ints(3, 4), 2, 1, 4)
    q, out = torch.zeros((2, 8, 192), dtype=torch.bfloat16), torch.zeros((2, 8, 128), dtype=torch.bfloat16)
    for args in ((c, Q.Kv8Step(ints(3), 1, 1, 4), h, q, out), (c, s, h, q.float(), out), (c, s, h, q[:1], out), (c, s, h, q[:, :4], out),
                 (c, s, h, q[:, :, :128], out), (c, s, h, q, out[:, :, :64]), (c, s, parts(latent=256)[1], q, out)):
        with pytest.raises(B.MoeError):
            L.attend(*args)
    with pytest.raises(B.MoeError):
        L.attend(c, s, h, q, out, form="none")
    for x in (torch.zeros((2, 512), dtype=torch.bfloat16), torch.zeros((1, 576), dtype=torch.bfloat16), torch.zeros((2, 576))):
        with pytest.raises(B.MoeError):
            L.append(c, s, x)
    with pytest.raises(B.MoeError):
        L.append(c, s, torch.zeros((2, 576), dtype=torch.bfloat16), norm=torch.zeros(256, dtype=torch.bfloat16))
    with pytest.raises(B.MoeError):
        L.LatentHeads(torch.zeros((8, 128, 512), dtype=torch.bfloat16), torch.zeros((4, 128, 512), dtype=torch.bfloat16))
    one = torch.zeros((1, 128, 512), dtype=torch.bfloat16)                    # a stride of 0 would stand for heads one behind the other
    for w_k, w_v in ((one.expand(8, 128, 512), one.repeat(8, 1, 1)), (one.repeat(8, 1, 1), one.expand(8, 128, 512))):
        with pytest.raises(B.MoeError):
            L.LatentHeads(w_k, w_v)
    with pytest.raises(B.MoeError):
        L.attend_workspace_bytes(c, s, h, "none")
    with pytest.raises(B.MoeError):
        L.LatentCache(torch.zeros((2, 8, 576), dtype=torch.bfloat16), 64, prefix=torch.zeros((3, 512), dtype=torch.bfloat16))
    both = torch.zeros((8, 256, 512), dtype=torch.bfloat16)                   # w_k and w_v as parts of one matrix
    h = L.LatentHeads(both[:, :128], both[:, 128:])
    assert h.c.w_k_head == h.c.w_v_head == 256 * 512


@pytest.mark.parametrize("change,status", [
    (dict(rot_dim=0), B.MOE_ERR_SHAPE), (dict(rot_dim=31), B.MOE_ERR_SHAPE), (dict(rot_dim=258), B.MOE_ERR_SHAPE),
    (dict(first=-1), B.MOE_ERR_INVALID_ARG), (dict(first=34), B.MOE_ERR_SHAPE), (dict(interleaved=2), B.MOE_ERR_INVALID_ARG),
    (dict(original_len=-1), B.MOE_ERR_INVALID_ARG), (dict(theta=0.0), B.MOE_ERR_INVALID_ARG), (dict(theta=math.inf), B.MOE_ERR_INVALID_ARG),
    (dict(factor=0.0), B.MOE_ERR_INVALID_ARG), (dict(factor=math.nan), B.MOE_ERR_INVALID_ARG), (dict(magnitude=math.inf), B.MOE_ERR_INVALID_ARG),
    (dict(original_len=100, high_turns=1.0), B.MOE_ERR_INVALID_ARG), (dict(original_len=100, low_turns=-1.0), B.MOE_ERR_INVALID_ARG),
])
def test_settings_of_the_rotation_are_checked(change, status):
    lib, r = P.load_library(), P.Rope(32)
    for k, v in change.items():
        setattr(r.c, k, v)
    rows = P.MoeRopeRows(16, 16, 1, 0, 64, 64, 64, 64)
    assert lib.moe_rope_rotate(None, r.ref, B.MOE_BF16, 2, 64, None, C.byref(rows), None) == status
    assert lib.moe_rope_last_error()


def test_rows_to_rotate_are_checked():
    lib, r = P.load_library(), P.Rope(32)
    x = torch.zeros((2, 2, 64), dtype=torch.bfloat16)

    def call(rows=2, hd=64, dtype=B.MOE_BF16, **change):
        s = P.MoeRopeRows(x.data_ptr(), x.data_ptr(), 2, 0, 128, 64, 128, 64)
        for k, v in change.items():
            setattr(s, k, v)
        return lib.moe_rope_rotate(None, r.ref, dtype, rows, hd, None, C.byref(s), None)

    assert call(dtype=2) == B.MOE_ERR_INVALID_ARG and call(rows=-1) == B.MOE_ERR_SHAPE and call(rows=(1 << 24) + 1) == B.MOE_ERR_SHAPE
    assert call(hd=1) == B.MOE_ERR_SHAPE and call(hd=1026) == B.MOE_ERR_SHAPE and call(hd=30) == B.MOE_ERR_SHAPE
    assert call(n_heads=-1) == B.MOE_ERR_SHAPE and call(n_heads=1025) == B.MOE_ERR_SHAPE and call(reserved=1) == B.MOE_ERR_INVALID_ARG
    assert call(in_row=-1) == B.MOE_ERR_INVALID_ARG
    assert call(out_row=127) == B.MOE_ERR_INVALID_ARG and b"overlap" in lib.moe_rope_last_error()
    assert call(in_row=256) == B.MOE_ERR_INVALID_ARG and b"same strides" in lib.moe_rope_last_error()
    assert call() == B.MOE_ERR_INVALID_ARG and b"not device memory" in lib.moe_rope_last_error()
    assert call(n_heads=0) == B.MOE_OK and call(rows=0) == B.MOE_OK           # nothing to do: no pointer is looked at
    assert lib.moe_rope_rotate(None, None, B.MOE_BF16, 2, 64, None, None, None) == B.MOE_ERR_INVALID_ARG
    assert lib.moe_rope_rotate(None, r.ref, B.MOE_BF16, 2, 64, None, None, None) == B.MOE_ERR_INVALID_ARG


def test_the_reference_against_hand_worked_values():
    x = torch.tensor([[[1.0, 0.0, 0.0, 2.0]]])
    quarter = R.rotate(x, torch.tensor([1]), rot=4, theta=1.0)                # every frequency 1: one radian
    assert torch.allclose(quarter, torch.tensor([[[math.cos(1), -2 * math.sin(1), math.sin(1), 2 * math.cos(1)]]], dtype=torch.float64))
    side = R.rotate(x, torch.tensor([1]), rot=2, theta=7.0, first=2, interleaved=True)
    assert torch.allclose(side, torch.tensor([[[1, 0, -2 * math.sin(1), 2 * math.cos(1)]]], dtype=torch.float64))
    assert R.frequencies(4, 100.0, factor=2.0) == [0.5, 0.05]
    # 2 pi positions: pair 0 turns once, pair 1 a tenth: low 0, high 1 keeps the first and squeezes nine tenths of the second
    w = R.frequencies(4, 100.0, factor=2.0, original_len=2 * math.pi, low=0.0, high=1.0)
    assert w[0] == 1.0 and abs(w[1] - 0.1 * (0.1 + 0.9 / 2)) < 1e-15
    rows = torch.zeros((1, 2, 3), dtype=torch.float64)
    rows[0, 0] = torch.tensor([1.0, 2.0, 3.0])
    rows[0, 1] = torch.tensor([0.0, 1.0, 0.0])
    q = torch.tensor([[[1.0, 0.0]]])                                          # one head: nope 1, rope 1
    w_k, w_v = torch.tensor([[[math.log(2.0), 0.0]]], dtype=torch.float64), torch.tensor([[[0.0, 3.0]]], dtype=torch.float64)
    out = R.attend(rows, q, w_k, w_v, [1], [0, 1], scale=1.0)[0]              # scores ln 2 and 0: weights 2/3, 1/3; values 6 and 3
    assert abs(out.item() - 5.0) < 1e-12
    out = R.attend(rows[:, 1:], q, w_k, w_v, [0], [0, 1], prefix=rows[0, :1], scale=1.0)[0]
    assert abs(out.item() - 5.0) < 1e-12
