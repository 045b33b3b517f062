"""Tiles of 64 rows: chunks over keys and values of 8 bits with a key head of up to 64 elements for each query head and few tokens a request."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import attention_plain as plain  # noqa: E402
from test_gpu_attention import BF, F16, TYPES  # noqa: E402
from test_gpu_attention8 import NAN_CODE, Paged8  # noqa: E402


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("heads,dim,page,block", [(3, 64, 16, 16), (8, 64, 8, 4), (5, 48, 64, 64), (2, 16, 1, 1)])
@pytest.mark.parametrize("window", [0, 1, 33, 1024])
def test_chunks_of_unlike_lengths(dtype, heads, dim, page, block, window):
    """63, 64 and 65 tokens, one, none, a chunk of several tiles; lengths in the cache that end anywhere."""
    lens, new = [1300, 1, 64, 65, 129, 0, 900, 1111, 63, 2, 500, 77], [250, 1, 64, 65, 63, 0, 1, 64, 63, 2, 31, 40]
    assert 16 * len(new) < sum(new) <= 64 * len(new)
    at = np.cumsum([0] + new)
    rows = sorted({int(x) for x in at[:-1]} | {int(x) - 1 for x in at[1:] if x} | {63, 64, 127, 128, 191, 192})
    Paged8(dtype, heads, heads, dim, page, block, lens, new, seed=window + dim, pad=2).check(window, [r for r in rows if r < sum(new)])


@pytest.mark.parametrize("n_req,most,dtype", [(445, 79, BF), (480, 79, F16), (600, 95, BF), (700, 127, F16), (1300, 79, BF)])
def test_many_requests(n_req, most, dtype):
    """As many as four workgroups on a CU have room for in LDS, more (tiles of 128 rows), more tiles than are shared out."""
    rng = np.random.default_rng(n_req)
    new = rng.integers(1, most + 1, n_req).tolist()
    p = Paged8(dtype, 2, 2, 32, 4, 4, [n + int(rng.integers(0, 200)) for n in new], new, seed=n_req)
    rows = sorted(set(rng.integers(0, sum(new), 60).tolist()) | {0, sum(new) - 1})
    p.check(rows=rows)
    p.check(window=50, rows=rows)


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("at", [0, 700, 1439])
def test_a_value_that_is_not_a_number(dtype, at):
    """Of the rows that see it those of its head have none; others, and those that a window takes past it, are what they are without it."""
    lens, new = [1500, 70, 5, 90], [120, 1, 5, 64]
    p = Paged8(dtype, 3, 3, 64, 16, 8, lens, new, seed=at)
    rows = [0, 5, 58, 59, 60, 63, 64, 119, 120, 125, 126, 189]
    want, want_window = p.want(rows=rows), p.want(window=100, rows=rows)
    page, place = p.place(0, at)
    p.v.view(torch.uint8)[page, place, 1, 3] = NAN_CODE
    for window, want in ((0, want), (100, want_window)):
        got = p.run(window)
        sees = [t for t in range(120) if 1380 + t >= at and (not window or 1380 + t - at < window)]
        hidden = torch.zeros_like(got[0], dtype=torch.bool)
        hidden[sees, 1, 3] = True
        assert got[0][hidden].isnan().all() and torch.isfinite(got[0][~hidden]).all()
        plain.check(got, {x: y for x, y in want.items() if x[0] not in sees}, window)
        assert torch.isfinite(got[1]).all() and not math.isnan(float(got[1].sum()))
