"""Elements that are not turned stay what they are, infinities among them."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2601_07048_amd import jx  # noqa: E402
from test_gpu_attention import TYPES, i32, normal  # noqa: E402


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("t", [3, 6000])
@pytest.mark.parametrize("dim,rot", [(64, 32), (64, 0), (128, 16)])
@pytest.mark.parametrize("pairs", [False, True])
def test_infinities_behind_the_turned_elements(dtype, t, dim, rot, pairs):
    heads, kv = 8, 2
    q, k, v = normal((t, heads, dim), dtype, 1), normal((t, kv, dim), dtype, 2), normal((t, kv, dim), dtype, 3)
    q[:, 1, rot + 3], q[:, 2, dim - 1], k[:, 1, rot + 9] = math.inf, -math.inf, math.inf
    cache = torch.zeros((2, t // 16 + 1, 16, kv, dim), dtype=dtype, device="cuda")
    angle = torch.rand((t, rot // 2)).cuda()
    cos, sin = (angle.cos(), angle.sin()) if rot else (None, None)
    slot = torch.arange(t, device="cuda")
    got = jx.qk_norm_rope(q, k, v, cache[0], cache[1], i32(list(range(t))), slot, cos, sin, interleaved=pairs)
    assert torch.equal(got[:, :, rot:], q[:, :, rot:])
    assert torch.equal(cache[0].flatten(0, 1)[:t, :, rot:], k[:, :, rot:])
    assert got[:, :, :rot].isfinite().all() and cache[0][..., :rot].isfinite().all()
