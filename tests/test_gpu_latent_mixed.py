"""A step of 1023 single tokens and one chunk of 4096 under 128 heads: the bounds are those of 1024 chunks."""
import pytest
import torch

from oracle import latent_ref as R
from paper_2502_06888_amd import binding as B
from paper_2502_06888_amd import kv8_binding as Q
from paper_2502_06888_amd import latent_binding as L
from test_gpu_latent import DEV, EXPANDED, ints, offsets_of, tolerance

pytestmark = pytest.mark.gpu


def test_single_tokens_beside_a_long_chunk():
    g = torch.Generator(device=DEV).manual_seed(1)
    n, heads, chunk, dims = 1024, 128, 4096, (128, 32, 32, 32)
    cached = [i % 60 for i in range(n)]
    new = [1] * n
    new[700] = chunk
    off = offsets_of(new)
    rows = torch.randn((n, chunk + 60, 160), generator=g, device=DEV, dtype=torch.bfloat16)
    w_k, w_v = (torch.randn((heads, 32, 128), generator=g, device=DEV, dtype=torch.bfloat16) * 128 ** -0.5 for _ in "kv")
    q = torch.randn((off[-1], heads, 64), generator=g, device=DEV, dtype=torch.bfloat16)
    out = torch.full((off[-1], heads, 32), -7.0, dtype=torch.bfloat16, device=DEV)
    cache, h = L.LatentCache(rows, 32), L.LatentHeads(w_k, w_v)
    step = Q.Kv8Step(ints(cached), off[-1], chunk, 59, row_offsets=ints(off))
    with pytest.raises(B.MoeError) as e:
        L.attend(cache, step, h, q, out, form="absorbed", workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    assert e.value.status == B.MOE_ERR_SHAPE and (out == -7.0).all()
    L.attend(cache, step, h, q, out)
    torch.cuda.synchronize()
    for seq, token in ((0, 0), (59, 0), (699, 0), (700, 0), (700, 1), (700, 2047), (700, 4095), (701, 0), (1023, 0)):
        row, sees = off[seq] + token, cached[seq] + token
        ref = R.attend(rows[seq:seq + 1].cpu(), q[row:row + 1].cpu(), w_k.cpu(), w_v.cpu(), [sees], [0, 1])
        err = (out[row:row + 1].cpu().double() - ref[0]).abs()
        assert (err <= tolerance(EXPANDED, *ref)).all()
