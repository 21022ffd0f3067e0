"""Steps of the latent cache whose launches would have 2^32 threads and more, and what the choice of form makes of them.  Sizes only: no GPU."""
import pytest
import torch

from paper_2502_06888_amd import binding as B
from paper_2502_06888_amd import kv8_binding as Q
from paper_2502_06888_amd import latent_binding as L


def sized(n_seq, max_len, heads, rows, new, cached, latent=512, nope=128, value=128, prefix=0):
    """A step's structs, of which only sizes are looked at."""
    cache = L.LatentCache.empty(1, 1, latent, 64, device="cpu")
    cache.n_seq = cache.c.n_seq = n_seq
    cache.c.max_len, cache.c.prefix_len = max_len, prefix
    ints = torch.zeros(n_seq + 1, dtype=torch.int32)
    step = Q.Kv8Step(ints[:n_seq], rows, new, cached, row_offsets=ints)
    h = L.LatentHeads(*(torch.zeros((heads, n, latent), dtype=torch.bfloat16) for n in (nope, value)))
    return cache, step, h


def workspace(args, form):
    """Bytes, or None where the call is refused for its workgroups."""
    try:
        return L.attend_workspace_bytes(*args, form)
    except B.MoeError as e:
        assert e.status == B.MOE_ERR_SHAPE and "workgroups" in e.message
        return None


MIXED = [
    # sequences, of which one brings a chunk of `new` tokens and the others one token each; 128 heads
    (1023, 4096, 4096), (1024, 4096, 4096), (1536, 4096, 4096), (512, 8192, 4096), (256, 16384, 4096),
]


@pytest.mark.parametrize("n_seq,new,cached", MIXED)
def test_absorbed_launches_of_2_to_the_32_threads_are_refused(n_seq, new, cached):
    """32 * 2 rows a workgroup of 512 threads: n_seq * ceil(new * 128 / 64) of them and more."""
    args = sized(n_seq, 32768, 128, n_seq - 1 + new, new, cached)
    groups = n_seq * -(-new * 128 // 64)
    assert (groups * 512 >= 2 ** 32) == (workspace(args, "absorbed") is None)


@pytest.mark.parametrize("n_seq,new,cached", MIXED)
def test_the_choice_of_form_takes_the_other_one_where_the_first_does_not_fit(n_seq, new, cached):
    args = sized(n_seq, 32768, 128, n_seq - 1 + new, new, cached)
    need = {form: workspace(args, form) for form in L.FORMS}
    assert need["expanded"] is not None
    assert need["auto"] == need["expanded"] or need["auto"] == need["absorbed"] is not None
    if need["absorbed"] is None:
        assert need["auto"] == need["expanded"]


def test_just_below_the_bound_both_forms_are_there():
    """1023 * 8190 workgroups of 512 threads: 2^32 less 512 * 10230."""
    args = sized(1023, 32768, 128, 1022 + 4095, 4095, 4096)
    assert 1023 * 8190 * 512 < 2 ** 32
    assert workspace(args, "absorbed") is not None and workspace(args, "expanded") is not None and workspace(args, "auto") is not None


def test_launches_that_bring_the_sums_out_of_the_latent_space():
    """finish_kernel: 512 threads for 32 rows of a head; 256 heads of 2^20 rows are 2^23 workgroups."""
    args = sized(4096, 512, 256, 1 << 20, 256, 100, latent=128, nope=32, value=32)
    assert workspace(args, "absorbed") is None                                # 4096 * ceil(256 * 256 / 64) = 2^22 of its attention would fit
    args = sized(4096, 512, 255, 1 << 20, 256, 100, latent=128, nope=32, value=32)
    assert workspace(args, "absorbed") is not None


def test_launches_that_make_keys_and_values():
    """expand_kernel: 128 * 4 threads for 128 slots of a sequence and some heads; 65536 sequences of 2^14 slots, a head at a time, are 2^23."""
    args = sized(65536, 1 << 14, 2, 65536, 1, (1 << 14) - 1)
    assert workspace(args, "expanded") is None
    args = sized(65535, 1 << 14, 2, 65535, 1, (1 << 14) - 129)
    assert workspace(args, "expanded") is not None
