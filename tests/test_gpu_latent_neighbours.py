"""The bits of a sequence's rows do not depend on what stands beside them: neighbours over the same prefix whose scores are huge or not
numbers, and rows that belong to no sequence."""
import pytest
import torch

from test_gpu_latent import FORMS, NAN, Layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("what", [1e8, 1e30, NAN, float("inf")])
def test_neighbours_with_scores_of_another_size(what, form):
    n = 64
    x = Layer(210, [7 * i % 90 for i in range(n)], [1] * n, 8, (128, 64, 32, 128), prefix=1500, std=8.0, tail=5)
    first = x.run(form)
    x.q[1::2] *= what                                                         # every other sequence, and the rows behind the last one
    x.q[n:] = what
    again = x.run(form)
    assert torch.equal(again[0:n:2], first[0:n:2])
