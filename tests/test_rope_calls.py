"""Calls of the rotation that the host refuses: rows of q and k in the same memory, a magnitude that 32 bits do not hold."""
import ctypes as C

import pytest
import torch

from paper_2502_06888_amd import binding as B
from paper_2502_06888_amd import rope_binding as P


@pytest.mark.parametrize("q,k", [((0, 0), (0, 0)), ((0, 1), (2, 1)), ((0, 1), (2, 0)), ((0, 1), (1, 2)), ((0, 0), (2, 0)), ((0, 1), (1, 1))])
def test_what_is_written_for_one_is_not_the_others(q, k):
    """(in, out) of each, by number of the tensor."""
    lib, t = P.load_library(), [torch.zeros((2, 2, 64), dtype=torch.bfloat16) for _ in range(3)]
    rows = [P.MoeRopeRows(t[a].data_ptr(), t[b].data_ptr(), 2, 0, 128, 64, 128, 64) for a, b in (q, k)]

    def call():
        return lib.moe_rope_rotate(None, P.Rope(32).ref, B.MOE_BF16, 2, 64, None, C.byref(rows[0]), C.byref(rows[1]))

    assert call() == B.MOE_ERR_INVALID_ARG and b"the same memory" in lib.moe_rope_last_error()
    rows[1].n_heads = 0                                                       # then nothing of k is looked at
    assert call() == B.MOE_ERR_INVALID_ARG and b"not device memory" in lib.moe_rope_last_error()


def test_both_may_be_read_from_one_tensor():
    lib, t = P.load_library(), [torch.zeros((2, 2, 64), dtype=torch.bfloat16) for _ in range(3)]
    rows = [P.MoeRopeRows(t[0].data_ptr(), t[i].data_ptr(), 2, 0, 128, 64, 128, 64) for i in (1, 2)]
    assert lib.moe_rope_rotate(None, P.Rope(32).ref, B.MOE_BF16, 2, 64, None, C.byref(rows[0]), C.byref(rows[1])) == B.MOE_ERR_INVALID_ARG
    assert b"not device memory" in lib.moe_rope_last_error()


@pytest.mark.parametrize("magnitude", [1e39, -1e300])
def test_a_magnitude_beyond_32_bits_is_refused(magnitude):
    lib, rows = P.load_library(), P.MoeRopeRows(16, 16, 1, 0, 64, 64, 64, 64)
    assert lib.moe_rope_rotate(None, P.Rope(32, magnitude=magnitude).ref, B.MOE_BF16, 2, 64, None, C.byref(rows), None) == B.MOE_ERR_INVALID_ARG
    assert b"magnitude" in lib.moe_rope_last_error()
