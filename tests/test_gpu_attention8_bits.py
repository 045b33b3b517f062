"""Codes as the 16-bit numbers that they stand for: attention of chunks over keys and values of 8 bits has the bits of attention over 16-bit keys and
values that are the same numbers, where both work on tiles of the same height; numbers at the lower end of what a type holds count."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2601_07048_amd import jx  # noqa: E402

import attention8_plain as plain8  # noqa: E402
import attention_plain as plain  # noqa: E402
from test_gpu_attention import BF, F16, TYPES, i32, normal  # noqa: E402
from test_gpu_attention8 import CODE, SCALE, Paged8  # noqa: E402


def elements(codes, scale, dtype):
    """The numbers, as 16-bit elements laid out as the codes are; all of them are such elements."""
    block = codes.shape[1] // scale.shape[1]
    x = codes.float() * scale.float().repeat_interleave(block, 1)[..., None]
    y = x.to(dtype)
    assert bool(((y.float() == x) | x.isnan()).all())
    return y


# query heads, key heads, dimension, page, block, lengths, new tokens: tiles of 128 rows, and of 256 (512 rows of one request, 2,048 of each of several)
CHUNKS = [(8, 2, 128, 16, 16, [333, 40], [100, 33]), (4, 1, 64, 16, 8, [900], [300]), (6, 3, 96, 64, 32, [700, 65, 1], [200, 65, 1]), (4, 4, 80, 4, 2, [190, 333], [64, 129]),
          (16, 2, 128, 1, 1, [60, 61], [40, 50]), (8, 2, 256, 16, 16, [300, 129], [129, 77]), (2, 1, 192, 32, 4, [500], [400]), (2, 2, 64, 16, 16, [500], [300]),
          (4, 1, 128, 16, 16, [2600], [2300]), (8, 1, 64, 64, 64, [1000], [700]), (2, 2, 96, 16, 8, [1500], [1300]), (16, 1, 48, 16, 1, [300, 200], [290, 140])]


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("heads,kv,dim,page,block,lens,new", CHUNKS)
def test_chunks_have_the_bits_of_16_bit_keys_and_values(dtype, heads, kv, dim, page, block, lens, new):
    p = Paged8(dtype, heads, kv, dim, page, block, lens, new, seed=dim + page, pad=1)
    k, v = elements(p.k, p.k_scale, dtype), elements(p.v, p.v_scale, dtype)
    for window in (0, 70, 1000):
        for scale in (p.scale, -0.3):
            p.scale = scale
            got = p.run(window)
            want = jx.paged_attention(p.q, k, v, p.table, p.q_start, p.kv_len, scale, window)
            assert torch.isfinite(got[0]).all()
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (window, scale)


def one_key(dtype, dim, new, byte, seed):
    """Requests of which each row sees a key of its own: the result is its value, whatever the weight's rounding."""
    n = 48
    p = Paged8(dtype, 4, 2, dim, 16, 1, [n + new - 1], [new], seed=seed, spare=1)
    g = torch.Generator().manual_seed(seed)
    for codes, scale in ((p.k, p.k_scale), (p.v, p.v_scale)):
        codes.view(torch.uint8).copy_(torch.randint(0, 256, codes.shape, generator=g).to(torch.uint8))
        codes.view(torch.uint8)[codes.float().isnan()] = 1
        scale.view(torch.uint8).copy_(byte(scale.shape, g))
    return p


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 40, 300])
def test_the_smallest_values(dtype, dim, new):
    """Scales from the smallest that a store leaves on (2^-126; binary16: those with codes that it holds), codes from the smallest on.  A row of one
    key has its value as it is, but for what the type does not hold."""
    low = 1 if dtype is BF else 127 - 15
    p = one_key(dtype, dim, new, lambda shape, g: torch.randint(low, low + 12, shape, generator=g).to(torch.uint8), seed=dim)
    p.k.view(torch.uint8).zero_()
    out, lse = p.run(window=1)
    value = plain8.stands_for(p.v, p.v_scale)
    last = int(p.kv_len)
    for i in range(new):
        page, place = p.place(0, last - new + i)
        want = value[page, place].repeat_interleave(2, 0)
        assert bool(((out[i].cpu().double() - want).abs() <= plain.TINY[dtype] / 2).all()), i
    p.check(rows=sorted({0, new // 2, new - 1}))


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("new", [1, 40, 300])
def test_the_smallest_keys(dtype, dim, new):
    """Keys of subnormal numbers that queries as large as the type has them, and the scale, bring back into the range of scores."""
    if dtype is BF:
        # keys of 2^-133 up to 2^-126 and a little, queries of 2^120: products from 2^-13 on
        p = one_key(dtype, dim, new, lambda shape, g: torch.randint(3, 5, shape, generator=g).to(torch.uint8), seed=dim)
        p.k.view(torch.uint8).bitwise_and_(0x8F)  # codes of up to 15 * 2^-9
        p.q = normal(p.q.shape, dtype, 3) * 2.0 ** 120
        p.scale = 2.0 ** 7
    else:
        p = one_key(dtype, dim, new, lambda shape, g: torch.randint(127 - 15, 127 - 13, shape, generator=g).to(torch.uint8), seed=dim)
        p.k.view(torch.uint8).bitwise_and_(0x8F)  # 2^-24 up to 2^-19
        p.q = normal(p.q.shape, dtype, 3) * 2.0 ** 10
        p.scale = 2.0 ** 6
    p.v_scale.view(torch.uint8).fill_(120)
    keys = plain8.stands_for(p.k, p.k_scale)
    assert float(keys.abs().max()) < (2.0 ** -125 if dtype is BF else 2.0 ** -18) and float(keys[keys != 0].abs().min()) >= plain.TINY[dtype]
    rows = sorted({0, 1, new // 2, new - 1} & set(range(new)))
    want = p.want(rows=rows)
    flat = plain.paged(p.q, torch.zeros_like(keys), plain8.stands_for(p.v, p.v_scale), p.table, p.q_start, p.kv_len, p.scale, 0, rows)
    assert any(abs(want[x][1] - flat[x][1]) > 16 * want[x][3] for x in want)  # lost keys would show
    plain.check(p.run(), want)
