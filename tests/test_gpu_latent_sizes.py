"""Attention over a latent cache where sizes lie far apart: tiles of very small, very large or no values, sums cut into ranges, queries and
keys that are tiny together, neighbours with scores of another size.  Bounds as in test_gpu_latent, whose absolute term (2^-100) is
replaced by half a step of the smallest numbers of bf16."""
import pytest
import torch

from paper_2502_06888_amd import latent_binding as L
from test_gpu_latent import DEV, EXPANDED, FORMS, Layer, tolerance

pytestmark = pytest.mark.gpu
DIMS = (128, 32, 32, 32)
TINY = 2.0 ** -134 - 2.0 ** -100


def on_device(x):
    """The layer's cache from its rows as they are now."""
    x.cache = L.LatentCache(x.rows.to(DEV), x.rope, None if x.prefix is None else x.prefix.to(DEV))
    return x


def check(got, form, ref):
    want = ref[0]
    there = ~want.isnan().all(-1).all(-1)
    err = (got.double() - want).abs()
    over = (err - tolerance(form, *ref) - TINY)[there]
    assert not over.isnan().any() and over.max() <= 0, f"over by {over.max():.3e} where the largest is {want[there].abs().max():.3e}"
    rel = (err[there].square().mean() / want[there].square().mean()).sqrt()
    assert rel <= 2.0 ** -8 * 0.65, f"off by {rel:.3e} in the mean"


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("sizes", [(0.0, 1e-6, 1e-6), (0.0, 1e-8, 1e-8), (1e-12, 0.0, 1e-12), (1e6, 1e-6, 1e-6), (1e-6, 1e6, 1.0), (1e-20, 1e-6, 1e-20)])
def test_tiles_of_no_values_and_of_sizes_far_apart(sizes, form):
    """A tile without values sets no scale for those behind it, and a tile of small ones keeps its bits behind larger ones."""
    x = Layer(201, [150, 130], [2, 3], 4, DIMS)
    for i, f in enumerate(sizes):
        x.rows[:, 64 * i:64 * (i + 1) if i < 2 else None, :128] *= f
    x.q[..., :32] /= max(sizes)
    check(on_device(x).run(form), form, x.reference())


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("sizes,low", [((1e6, 1e-6, 1e-6), 0), ((1e-6, 1e6, 1e-6), 1), ((1e-6, 1e-6, 1e20), 2), ((1e20, 1.0, 1e-20), 0)])
def test_tiles_that_hardly_count_set_no_scale(sizes, low, form):
    """Large values whose weights are about e^-300 of the others': what remains are the small ones."""
    x = Layer(202, [150, 140], [2, 3], 4, DIMS)
    at = [slice(0, 64), slice(64, 128), slice(128, None)]
    for i, f in enumerate(sizes):
        x.rows[:, at[i], :128] *= f
        x.rows[:, at[i], 128:] = -60.0 if i == low else 0.0
    x.q[..., :32] /= max(sizes)
    x.q[..., 32:] = 1.25
    check(on_device(x).run(form), form, x.reference())


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("size", [1e34, 1e-24])
def test_sums_in_ranges_of_values_of_any_size(size, form):
    """Positive values under nearly equal scores: the sum of a range is far larger than its mean."""
    x = Layer(203, [5000, 17], [1, 2], 4, DIMS, prefix=3001, max_len=5100)
    for rows in (x.rows, x.prefix):
        rows[..., :128] = rows[..., :128].abs() * size
    x.w_v = x.w_v.abs()
    x.h = L.LatentHeads(x.w_k.to(DEV), x.w_v.to(DEV))
    x.q[..., :32] /= size
    check(on_device(x).run(form), form, x.reference())


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("q,latents", [(1e-20, 1e-20), (1e-25, 1e-25), (1e-14, 1e-25), (1e25, 1e-25), (1e-25, 1e25), (3e-38, 1.0), (1e-38, 1e30)])
def test_queries_and_latents_of_any_size(q, latents, form):
    """Small or large together, beside a part with the position that is neither, in tiles of which rows see a part."""
    x = Layer(204, [10, 90, 0], [60, 3, 70], 4, DIMS)
    x.rows[..., :128] *= latents
    x.q[..., :32] *= q
    check(on_device(x).run(form), form, x.reference())


@pytest.mark.parametrize("form", [EXPANDED])
@pytest.mark.parametrize("q,latents", [(1.0, 1e-30), (1e-10, 1e-30)])
def test_latents_whose_shares_are_below_the_absorbed_forms_range(q, latents, form):
    x = Layer(205, [10, 90, 0], [60, 3, 70], 4, DIMS)
    x.rows[..., :128] *= latents
    x.q[..., :32] *= q
    check(on_device(x).run(form), form, x.reference())


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("sizes", [(1e20, 1e-20, 1e-20), (1e-20, 1e20, 1e-20), (1e18, 0.0, 1e-18)])
def test_tiles_beyond_what_sums_can_hold_beside_each_other(sizes, form):
    """Under queries as small as the smallest keys, sums of a large tile with those of one less than 2^-100 of it."""
    test_tiles_of_no_values_and_of_sizes_far_apart(sizes, form)


@pytest.mark.parametrize("cached,prefix", [([100, 700], 200), ([30, 5], 0)])
def test_the_smallest_values(cached, prefix):
    """Values of 2^-120 to 2^-119, each one latent, so that no product on the way is smaller."""
    x = Layer(206, cached, [40, 2], 4, DIMS, prefix=prefix)
    one = torch.eye(32, 128, dtype=torch.bfloat16)
    x.w_k = x.w_v = one.expand(4, 32, 128).contiguous()
    x.h = L.LatentHeads(x.w_k.to(DEV), x.w_v.to(DEV))
    g = torch.Generator().manual_seed(7)
    for rows in [x.rows] if prefix == 0 else [x.rows, x.prefix]:
        rows[..., :128] = (1 + torch.randint(0, 128, rows[..., :128].shape, generator=g) / 128).to(torch.bfloat16) * 2.0 ** -120
    check(on_device(x).run(EXPANDED), EXPANDED, x.reference())
