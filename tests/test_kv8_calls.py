"""Calls of the 8-bit key-value cache that the host decides on its own: streams of workspaces, sizes and strides that are
accepted or refused.  No GPU needed."""
import contextlib

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
    for call, _ in calls[:3]:                                                  # nothing on the current stream
        used.clear()
        call(None)
        assert not used
