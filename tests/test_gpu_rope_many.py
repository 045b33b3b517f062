"""Norm, rotation and store of so many rows that a group of lanes takes four heads of a token: last groups of one, two and three
rows, groups over queries, keys and values, padding, queries in place.  Bounds: those of rope_plain."""
import pytest
import torch

pytestmark = pytest.mark.gpu

import attention_plain as plain  # noqa: E402
from paper_2601_07048_amd import jx  # noqa: E402
from test_gpu_attention import TYPES, normal, rope_plain  # noqa: E402


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("heads,kv", [(7, 1), (6, 2), (9, 3), (8, 4), (2, 1), (3, 3)])
@pytest.mark.parametrize("dim,rot,pairs", [(64, 64, False), (56, 32, True), (128, 64, True), (80, 80, False), (256, 256, False), (192, 0, False)])
@pytest.mark.parametrize("normed", [False, True])
def test_four_heads_a_group(dtype, heads, kv, dim, rot, pairs, normed):
    lanes = 8 if dim <= 64 else 16 if dim <= 128 else 32
    t = 524288 // (lanes * (heads + 2 * kv)) + 37
    q, k, v = normal((t, heads, dim), dtype, 1, 2.0), normal((t, kv, dim), dtype, 2, 2.0), normal((t, kv, dim), dtype, 3)
    page, n_pos = 16, t
    pages = t // page + 3
    cache = normal((2, pages, page, kv, dim), dtype, 5)
    before = cache.clone()
    g = torch.Generator().manual_seed(t)
    pos, slot = torch.randperm(n_pos, generator=g).int(), torch.randperm(pages * page, generator=g)[:t]
    pos[t - 20:], slot[t - 20:] = -1, -1  # padding
    slot[5] = pages * page
    pos[6] = n_pos
    angle = torch.rand((n_pos, rot // 2), generator=g) * 6.3
    cos, sin = (angle.cos().cuda(), angle.sin().cuda()) if rot else (None, None)
    wq, wk = (normal((dim,), dtype, 6), normal((dim,), dtype, 7)) if normed else (None, None)
    at = pos.long().clamp(0, n_pos - 1)
    turn = (cos.cpu()[at], sin.cpu()[at]) if rot else (None, None)
    want_q, want_k = (rope_plain(x.cpu(), w.cpu() if normed else None, 1e-6, *turn, pairs) for x, w in ((q, wq), (k, wk)))
    got = jx.qk_norm_rope(q, k, v, cache[0], cache[1], pos.cuda(), slot.cuda(), cos, sin, wq, wk, eps=1e-6, interleaved=pairs, out=q)
    assert got is q
    here = (pos >= 0) & (pos < n_pos) if rot else pos >= 0
    stored = here & (slot >= 0) & (slot < pages * page)
    u, tiny = plain.UNIT[dtype], plain.TINY[dtype]

    def close(a, want, rows):
        y, bound = want
        assert bool(((a.cpu().double() - y[rows]).abs() <= (bound[rows] + u * y[rows].abs()) * 1.01 + tiny / 2).all())

    close(q.cpu()[here], want_q, here)
    assert not q.cpu()[~here].any()
    flat = cache.flatten(1, 2).cpu()
    close(flat[0][slot[stored]], want_k, stored)
    assert torch.equal(flat[1][slot[stored]], v.cpu()[stored])
    others = torch.ones(pages * page, dtype=torch.bool)
    others[slot[stored]] = False
    assert torch.equal(flat[:, others], before.flatten(1, 2).cpu()[:, others])
