"""The store into blocks of 8 bits where a team of lanes takes several runs of rows in turn: so many tokens and key heads that there are more teams
than the card holds wavefronts a few times.  Teams of a wavefront and of a workgroup, one to eight rows a lane."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from test_gpu_attention import BF, F16  # noqa: E402
from test_gpu_attention8 import check_store, flat, run_store, store_case  # noqa: E402


def lanes_of(dim, block):
    return (8 if dim <= 64 else 16 if dim <= 128 else 32) * block


def several(tokens, kv, dim, block):
    """Whether a team takes several runs."""
    lanes = lanes_of(dim, block)
    return lanes >= 64 and tokens * kv * (4 if lanes > 256 else 1) > 32768


def spans(tokens, block, rng):
    """Chunks of one token up to a few blocks, from places all over a block on, one long one among them."""
    out = [(3, 9 * block + 5)]
    while sum(n for _, n in out) < tokens:
        out.append((int(rng.integers(0, 4 * block)), int(rng.choice([1, 2, 3, block - 1, block, block + 1, 2 * block + 3, int(rng.integers(1, 3 * block + 2))])) or 1))
    return out


def uneven(c, rng, block, dtype):
    """Sizes that differ from token to token, so that neighbouring blocks have scales far apart, and within one the largest is anywhere; rows that are not
    stored, at the end of a chunk and as whole chunks; blocks of zeros and single values that are not finite."""
    t = len(c["pos"])
    low, high = (-40, 40) if dtype is BF else (-9, 9)
    for name in ("k", "v"):
        x = c[name]
        x *= torch.exp2(torch.from_numpy(rng.integers(low, high, (t, x.shape[1], 1)).astype(np.float32))).to(dtype).cuda()
        x[torch.from_numpy(rng.random(t) < 0.02).cuda()] = 0
        if name == "v" or c["wk"] is None:  # a norm would spread them over the row
            x[int(rng.integers(t)), -1, 3], x[int(rng.integers(t)), 0, 5], x[int(rng.integers(t)), 0, 1] = float("nan"), float("inf"), -float("inf")
    ends = [i for i in range(t) if i + 1 == t or c["slot"][i + 1] != c["slot"][i] + 1 and c["pos"][i + 1] != c["pos"][i] + 1]
    for i in rng.choice(ends, 12, replace=False):
        if rng.random() < 0.5:
            c["slot"][i] = -1
        else:
            c["pos"][i] = -1
    begins = [0] + [i + 1 for i in ends[:-1]]
    for j in rng.choice(len(ends), 5, replace=False):
        for i in range(begins[j], ends[j] + 1):
            c["slot"][i] = -1
    return c


CASES = [(BF, 64, 8, 8, 16), (F16, 64, 8, 16, 16), (BF, 64, 8, 32, 32), (F16, 48, 3, 64, 64), (F16, 128, 8, 4, 16), (BF, 128, 8, 8, 8), (F16, 128, 8, 16, 64), (BF, 128, 2, 32, 32),
         (F16, 128, 4, 32, 128), (BF, 112, 3, 64, 64), (BF, 256, 8, 2, 4), (F16, 256, 8, 4, 4), (BF, 256, 8, 8, 64), (F16, 256, 2, 16, 16), (BF, 208, 3, 32, 32),
         (F16, 192, 2, 64, 64), (BF, 256, 2, 64, 128)]


@pytest.mark.parametrize("dtype,dim,kv,block,page", CASES)
@pytest.mark.parametrize("normed", [False, True])
def test_several_runs_of_a_team(dtype, dim, kv, block, page, normed):
    rng = np.random.default_rng(dim + block)
    tokens = 32768 // kv // (4 if lanes_of(dim, block) > 256 else 1) + 37
    c = store_case(dtype, spans(tokens, block, rng), kv, kv, dim, 0 if dim == 112 or not normed else 32, page, block, block % 3 == 1, normed, seed=block)
    assert several(len(c["pos"]), kv, dim, block)
    check_store(uneven(c, rng, block, dtype))


@pytest.mark.parametrize("dtype,dim,kv,block,page", [x for x in CASES if x[3] in (8, 16, 32, 64)])
def test_one_run_or_several(dtype, dim, kv, block, page):
    """What a team stores beside others is what it stores alone: bit for bit the chunks of a step, in steps of their own."""
    rng = np.random.default_rng(dim + block + 1)
    tokens = 32768 // kv // (4 if lanes_of(dim, block) > 256 else 1) + 37
    at = spans(tokens, block, rng)
    c = store_case(dtype, at, kv, kv, dim, 32, page, block, False, True, seed=block + 1)
    uneven(c, rng, block, dtype)
    first = {x: c[x].view(torch.uint8).clone().view(c[x].dtype) for x in ("k_cache", "v_cache", "k_scale", "v_scale")}
    whole = run_store(c).clone()
    held = flat(c["k_cache"], c["k_scale"]), flat(c["v_cache"], c["v_scale"])
    for x, y in first.items():
        c[x].view(torch.uint8).copy_(y.view(torch.uint8))
    cut, i = [0], 0
    for _, n in at:  # steps of whole chunks, each of too few tokens for several runs
        i += n
        if i - cut[-1] >= tokens // 5 or i == len(c["pos"]):
            cut.append(i)
    assert len(cut) > 4
    for a, b in zip(cut, cut[1:]):
        assert not several(b - a, kv, dim, block)
        part = dict(c, **{x: c[x][a:b] for x in ("q", "k", "v")}, pos=c["pos"][a:b], slot=c["slot"][a:b])
        assert torch.equal(run_store(part), whole[a:b])
    again = flat(c["k_cache"], c["k_scale"]), flat(c["v_cache"], c["v_scale"])
    for x, y in zip(held, again):
        assert torch.equal(x[0].view(torch.uint8), y[0].view(torch.uint8)) and torch.equal(x[1], y[1])
