"""Scales next to 0 and 0 itself, beside products of queries and keys that are large."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from test_gpu_attention import BF, Paged  # noqa: E402


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("lens", [[200], [3000]])
@pytest.mark.parametrize("scale,size", [(0.0, 1e14), (-0.0, 1e15), (1e-33, 1e16), (-2e-37, 1e18), (1e-30, 1e14)])
def test_small_scales_of_large_products(new, lens, scale, size):
    p = Paged(BF, 4, 2, 64, 16, lens, [new], seed=3)
    p.q, p.k = (p.q.float() * size).to(BF), (p.k.float() * size).to(BF)
    p.scale = scale
    p.check(rows=[0, new - 1])
