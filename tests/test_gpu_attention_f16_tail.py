"""binary16: one key with nearly all the weight, and a long tail of others that each have next to none but count together.

Bound.  Weights are rounded to binary16 2^7 times as large as they are beside the running maximum, so that half the type's smallest
step, 2^-25, is 2^-32 of the largest weight: n keys add at most 2^-32 sum_j |v_j|, in place of tiny / 2 sum_j |v_j| among the bounds
of attention_plain."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import attention_plain as plain  # noqa: E402
from test_gpu_attention import F16, Paged  # noqa: E402


@pytest.mark.parametrize("below", [12.0, 18.0, 21.0], ids=lambda x: f"{x:.0f} nats")
@pytest.mark.parametrize("tokens,page", [(1, 16), (3, 16), (3, 8)], ids=["16 rows", "32 rows", "128 rows"])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_long_tail_counts(below, tokens, page, dim):
    """Of more than 1,024 requests each one's keys are taken in one go, so that all of the tail stands beside the first key."""
    n, others = 60000, 1030
    p = Paged(F16, 8, 1, dim, page, [n] + [4] * others, [tokens] * (1 + others), seed=dim, spare=0)
    p.scale = 1.0
    at = p.table[0, :n // page].long()
    k, v = p.k[at].flatten(0, 1).clone(), p.v[at].flatten(0, 1).clone()
    k[:, 0, 0] = -below
    k[0] = 0
    v.abs_()
    v[0] = 0
    p.k[at], p.v[at] = k.unflatten(0, (-1, page)), v.unflatten(0, (-1, page))
    p.q.mul_(0.02)
    p.q[:tokens, :, 0] = 1
    out, lse = p.run()
    k, v = k[:, 0].cpu().double(), v[:, 0].cpu().double()
    for t in range(tokens):
        seen = n - tokens + 1 + t
        for h in (0, 5):
            o, l, bo, bl = plain.attend_row(p.q[t, h].cpu().double(), k[:seen], v[:seen], 1.0, F16, rounded=False)
            w = torch.exp(k[:seen] @ p.q[t, h].cpu().double() - l)
            bo = bo + (plain.UNIT[F16] * (w @ v[:seen]) + 2.0 ** -32 * v[:seen].sum(0)) * 1.02
            err = (out[t, h].cpu().double() - o).abs()
            assert bool((err <= bo).all()), (t, h, float((err / o).max()))
            assert abs(float(lse[t, h]) - l) <= bl
    assert out.isfinite().all() and math.isfinite(float(lse.sum()))


@pytest.mark.parametrize("tokens,page", [(1, 16), (3, 16), (3, 8)], ids=["16 rows", "32 rows", "128 rows"])
def test_weights_at_the_top_of_their_range(tokens, page):
    """Scores that rise by just under 2^8 over the running maximum, which then stays: weights of up to 2^15 times values near the
    type's largest, and sums of them, stay numbers."""
    n = 400
    p = Paged(F16, 8, 1, 64, page, [n] + [4] * 1030, [tokens] * 1031, seed=1, spare=0)
    at = p.table[0, :n // page].long()
    k = torch.zeros((n, 64), dtype=F16, device="cuda")
    k[64:, 0] = 7.99 * math.log(2.0)
    p.k[at], p.v[at] = k.unflatten(0, (-1, page))[:, :, None], torch.full_like(p.v[at], 60000.0)
    p.q.zero_()
    p.q[:tokens, :, 0] = 1
    p.scale = 1.0
    p.check(rows=list(range(tokens)))
