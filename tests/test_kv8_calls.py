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
