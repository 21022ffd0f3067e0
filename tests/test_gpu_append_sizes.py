"""Normalised latents of the cache's append where squares leave the range of 32 bits."""
import pytest
import torch

from oracle import latent_ref as R
from paper_2502_06888_amd import kv8_binding as Q
from paper_2502_06888_amd import latent_binding as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dims", [(512, 64), (256, 32), (128, 64)])
@pytest.mark.parametrize("size,eps", [(1e18, 1e-6), (1e20, 1e-6), (1e38, 0.0), (1e-12, 1e-30), (1e-20, 0.0), (1e-25, 1e-38), (1e-37, 0.0), (1e-25, 1e-6)])
def test_rows_of_any_size_are_normalised(size, eps, dims):
    g = torch.Generator().manual_seed(5)
    latent, width = dims[0], sum(dims)
    x = (torch.randn((6, width), generator=g).clamp(-3, 3) * size).to(torch.bfloat16)
    x[2, :latent] = 0
    x[2, 5] = size                                                            # one element has it all
    w = torch.randn(latent, generator=g).to(torch.bfloat16)
    cache = L.LatentCache(torch.zeros((1, 8, width), dtype=torch.bfloat16, device=DEV), dims[1])
    offsets = torch.tensor([0, 6], dtype=torch.int32, device=DEV)
    step = Q.Kv8Step(torch.zeros(1, dtype=torch.int32, device=DEV), 6, 6, 0, row_offsets=offsets)
    L.append(cache, step, x.to(DEV), norm=w.to(DEV), eps=eps)
    want = torch.zeros((1, 8, width), dtype=torch.float64)
    R.append(want, x, [0], [0, 6], latent, w, torch.tensor(eps, dtype=torch.float32).item())
    # half a step of bf16, sums and products in 32 bits; half a step of its smallest numbers
    tol = (2.0 ** -8 + 2.0 ** -18) * want.abs() + 2.0 ** -134
    assert ((cache.rows.cpu().double() - want).abs() <= tol).all()
