"""Calls of the 8-bit key-value cache that the host decides on its own: streams of workspaces, sizes and strides that are
accepted or refused.  No GPU needed."""
import contextlib
import os
import re

import pytest
import torch

from paper_2502_06888_amd import attn_binding as A
from paper_2502_06888_amd import binding as B
from paper_2502_06888_amd import kv8_binding as Q


def cache(n_seq=2, kv=2, hd=64, max_len=128, block=32):
    return Q.Kv8Cache.empty(n_seq, kv, hd, max_len, block, device="cpu")


def ints(*v):
    return torch.tensor(v, dtype=torch.int32)


class FakeStream:
    cuda_stream = 0


class ForeignStream:
    """In the place of torch.cuda.ExternalStream, which takes a device to make."""
    cuda_stream = 0


@pytest.fixture
def current(monkeypatch):
    """The stream that is current when a workspace is made, for each one made."""
    streams, made = [None], []

    @contextlib.contextmanager
    def enter(stream):
        streams.append(stream)
        yield
        streams.pop()

    def noting(f):
        def g(*a):
            made.append(streams[-1])
            return f(*a)
        return g

    monkeypatch.setattr(torch.cuda, "stream", enter)
    for name in ("attend_workspace", "evict_workspace"):
        monkeypatch.setattr(Q, name, noting(getattr(Q, name)))
    return made


def test_a_workspace_made_by_a_call_belongs_to_its_stream(current):
    c, s, st = cache(max_len=4096), Q.Kv8Step(ints(3, 4), 2, 1, 4000), FakeStream()
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    w = torch.zeros((2, 2, 4096))
    for stream in (st, None):
        with contextlib.suppress(B.MoeError, RuntimeError, AssertionError):     # host tensors: refused by the library
            Q.attend(c, s, q, q.clone(), stream=stream)
        with contextlib.suppress(B.MoeError, RuntimeError, AssertionError):
            Q.evict(c, ints(3, 4), 4, 32, 0, None, w, stream=stream)
    assert current == [st, st, None, None]


def test_the_workspace_of_the_layer_belongs_to_the_compute_stream(current):
    ctx = object.__new__(A.AttnContext)
    ctx.h, ctx.compute, ctx.cfg = None, FakeStream(), A.MoeAttnConfig(256, 4, 2, 64, 8, 1, 1, 0, 1e4, 1e-5)
    ctx.kv8_workspace(cache(max_len=4096), Q.Kv8Step(ints(3, 4), 2, 1, 4000), True)
    assert current == [ctx.compute]


def test_tensors_of_a_call_on_another_stream_are_recorded_on_it(monkeypatch):
    """A caller may drop its tensors behind the call: each one's memory waits for the stream."""
    used = []
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, s: used.append((t.data_ptr(), s)))
    monkeypatch.setattr(Q, "_check", lambda status: None)                      # host tensors: refused by the library
    monkeypatch.setattr(A, "_check", lambda status, ctx=None: None)
    monkeypatch.setattr(Q, "_stream", lambda cache, stream: 0)
    monkeypatch.setattr(torch.cuda, "ExternalStream", ForeignStream)
    c, st = cache(), FakeStream()
    s = Q.Kv8Step(ints(3, 4), 2, 1, 4, row_offsets=ints(0, 1, 2), next_position=ints(3, 4))
    x = [torch.zeros((2, n, 64), dtype=torch.bfloat16) for n in (2, 2, 4, 4)]
    w, p, h = [torch.zeros((2, 2, 128)) for _ in range(2)], torch.zeros((2, 2, 128), dtype=torch.int32), ints(40, 4)
    kept, nxt = torch.zeros((2, 2, 32), dtype=torch.int32), ints(40, 4)
    space = torch.empty(1 << 16, dtype=torch.uint8)
    both = [c.k, c.v, c.k_scale, c.v_scale, c.position, s.cached, s.row_offsets, s.next_position]
    ctx = object.__new__(A.AttnContext)
    ctx.h, ctx.compute, ctx.lib, ctx.cfg = None, st, A.load_library(), A.MoeAttnConfig(256, 4, 2, 64, 8, 1, 1, 0, 1e4, 1e-5)
    rows = [torch.zeros((2, 256), dtype=torch.bfloat16) for _ in range(2)]
    calls = [(lambda t: Q.append(c, s, x[0], x[1], stream=t), both + x[:2]),
             (lambda t: Q.attend(c, s, x[2], x[3], w[0], w[1], space, stream=t), both + x[2:] + w + [space]),
             (lambda t: Q.evict(c, h, 40, 32, 0, nxt, w[0], w[1], p, kept, space, stream=t), both[:5] + w + [h, nxt, p, kept, space]),
             (lambda t: ctx.forward_kv8(c, s, rows[0], rows[1], space, weight_in=w[0], weight_out=w[1]), both + rows + w + [space])]
    for call, tensors in calls:
        used.clear()
        call(st)
        assert sorted(used, key=lambda u: u[0]) == sorted(((t.data_ptr(), st) for t in tensors), key=lambda u: u[0])
    for call, _ in calls[:3]:                                                  # nothing on the current stream, or on one that
        for stream in (None, ForeignStream()):                                 # may end before the tensors do
            used.clear()
            call(stream)
            assert not used


@pytest.mark.parametrize("seqs,kv,heads,hd,rows,new,cached,max_len", [
    (512, 8, 32, 128, 512 + 1024, 1024, 512, 2048),     # one chunk of a prompt among single tokens
    (512, 8, 32, 128, 512 + 1024, 1025, 512, 2048),
    (64, 8, 32, 128, 64 * 8192, 8192, 0, 8192),         # 64 long prompts
    (64, 8, 32, 128, 1 << 20, 16384, 0, 16384),
    (256, 8, 32, 128, 4096, 2048, 0, 4096),
    (65536, 8, 64, 32, 1 << 20, 17, 100, 128),
    (1, 1, 8, 128, 1 << 20, 1 << 20, 0, 1 << 20),
])
def test_steps_whose_launches_fit_are_accepted(seqs, kv, heads, hd, rows, new, cached, max_len):
    """The limit is one of workgroups, of 128 rows each, not of the rows that the bounds allow every sequence."""
    c = cache(kv=kv)
    c.c.n_seq, c.c.n_kv_heads, c.c.head_dim, c.c.max_len, c.c.block = seqs, kv, hd, max_len, 64
    s = Q.Kv8Step(ints(0), rows, new, cached, row_offsets=ints(0, 1))
    assert 0 <= Q.attend_workspace_bytes(c, s, heads, False) <= Q.attend_workspace_bytes(c, s, heads, True)


def test_the_limit_of_a_launch_is_the_documented_one():
    """Tiles of 128 rows per pair, and slots / 128 where weights are summed."""
    most = (1 << 24) - 1
    c = cache(kv=16)
    for seqs, kv, heads, max_len in ((64, 16, 64, 1 << 18), (65536, 16, 128, 1 << 11), (4096, 16, 16, 1 << 16), (3, 16, 64, 1 << 20),
                                     (700, 16, 32, 1 << 17), (1, 1, 8, 1 << 20), (256, 1, 8, 1 << 20), (30, 8, 64, 1 << 20)):
        c.c.n_seq, c.c.n_kv_heads, c.c.max_len = seqs, kv, max_len
        pairs, g = seqs * kv, heads // kv
        for new in (1, 16, 17, 300, 4000, 70000, 1 << 20):
            for cached in (0, 3, max_len // 2, max_len):
                for rows in {1, new // 2 + 1, new, min(seqs * new, 1 << 20)}:
                    if new > max_len:
                        continue
                    s = Q.Kv8Step(ints(0), rows, new, cached, row_offsets=ints(0, 1))
                    fits = pairs * -(-min(new, rows) * g // 128) <= most
                    sums = pairs * -(-min(new + cached, max_len) // 128) <= most
                    if fits:
                        assert Q.attend_workspace_bytes(c, s, heads, False) >= 0
                        assert not sums or Q.attend_workspace_bytes(c, s, heads, True) >= 0
                    if not sums:
                        with pytest.raises(B.MoeError) as e:
                            Q.attend_workspace_bytes(c, s, heads, True)
                        assert e.value.status == B.MOE_ERR_SHAPE and "workgroups" in e.value.message


def attend_strides(c, s, heads, row, head):
    """Text of what moe_kv8_attend says to host tensors with these strides of out: it asks for device memory after the strides."""
    x = torch.zeros(8, dtype=torch.bfloat16)
    assert Q.load_library().moe_kv8_attend(None, c.ref, s.ref, heads, x.data_ptr(), 256, 64, 0.0, x.data_ptr(), row, head, None, None, None, 0) == B.MOE_ERR_INVALID_ARG
    return Q.load_library().moe_kv8_last_error()


def test_outputs_are_refused_if_and_only_if_pieces_share_an_element():
    for rows, heads, hd in ((2, 2, 64), (2, 4, 64), (3, 2, 32), (7, 4, 32), (5, 6, 64), (1, 4, 32), (9, 2, 128), (1, 2, 128)):
        c, s = cache(n_seq=rows, kv=2, hd=hd), Q.Kv8Step(ints(*[3] * rows), rows, 1, 4)
        for row in range(0, 6 * hd * heads // 4, 8):
            for head in range(0, 6 * hd * rows // 4, 24):
                starts = sorted(r * row + h * head for r in range(rows) for h in range(heads))
                share = any(b - a < hd for a, b in zip(starts, starts[1:]))
                assert (b"overlap" in attend_strides(c, s, heads, row, head)) == share, (rows, heads, hd, row, head)


def test_strides_of_any_size_are_judged():
    c, s = cache(), Q.Kv8Step(ints(3, 4), 2, 1, 4)
    far = 1 << 62
    for row, head, share in ((far, 64, False), (64, far, False), (far, far, True), (far, far - 64, False), (far, far - 56, True)):
        assert (b"overlap" in attend_strides(c, s, 2, row, head)) == share


def test_nothing_is_asked_of_q_and_out_where_there_are_no_rows():
    c, lib = cache(), Q.load_library()
    s = Q.Kv8Step(ints(3, 4), 0, 0, 4, row_offsets=ints(0, 0, 0))
    for p in (None, torch.zeros(8, dtype=torch.bfloat16).data_ptr()):
        assert lib.moe_kv8_attend(None, c.ref, s.ref, 4, p, 0, 0, 0.0, p, 0, 0, None, None, None, 0) == B.MOE_ERR_INVALID_ARG
        assert b"cache.k is not device memory" in lib.moe_kv8_last_error()


def test_assembly_that_writes_m0_names_it():
    """The compiler is told of every register that inline assembly overwrites."""
    folder = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_06888_amd", "csrc")
    found = 0
    for name in sorted(n for n in os.listdir(folder) if n.endswith((".hip", ".h"))):
        for text in re.findall(r"asm volatile\((.*?)\);\n", open(os.path.join(folder, name)).read(), flags=re.S):
            code, _, rest = text.partition('" ::')
            if re.search(r"\bm0\b", code):
                found += 1
                assert '"m0"' in rest, text
    assert found >= 3
