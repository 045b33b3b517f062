"""What is not a number and is seen reaches the result, whoever takes the keys: a wavefront, a workgroup or several."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import attention_plain as plain  # noqa: E402
from test_gpu_attention import BF, F16, Paged  # noqa: E402


@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("new", [1, 3, 40])
@pytest.mark.parametrize("lens", [[60], [250], [3000], [700, 64, 5000, 130]], ids=["unit", "own", "one", "unlike"])
def test_a_query_that_is_not_a_number(dtype, new, lens):
    p = Paged(dtype, 4, 2, 128, 16, lens, [min(new, n) for n in lens], seed=new)
    rows = p.q.shape[0]
    bad = sorted({0, rows // 2, rows - 1})
    p.q[bad, 1, 5] = math.nan
    out, lse = p.run()
    assert out[bad, 1].isnan().all() and lse[bad, 1].isnan().all()
    want = p.want(rows=bad)
    plain.check((out, lse), {at: w for at, w in want.items() if at[1] != 1})
    out[bad, 1], lse[bad, 1] = 0, 0
    assert out.isfinite().all() and lse.isfinite().all()


@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("new", [1, 3, 40])
@pytest.mark.parametrize("where", ["keys", "values"])
@pytest.mark.parametrize("length,first", [(250, 64), (3000, 0), (3000, 1984), (3000, 2944), (20000, 6400)])
def test_keys_and_values_that_are_not_numbers_over_a_whole_part(dtype, new, where, length, first):
    """64 keys in a row, as many as a part of a request has at the least; all new tokens stand behind them or among them."""
    p = Paged(dtype, 4, 2, 64, 16, [length], [new], seed=first)
    cache = p.k if where == "keys" else p.v
    end = min(first + 64, length - new + 1)  # so that every row sees them
    for j in range(first, end):
        cache[int(p.table[0, j // 16]), j % 16, 1, 7] = math.nan
    out, lse = p.run()
    plain.check((out, lse), {at: w for at, w in p.want(rows=[0, new - 1]).items() if at[1] < 2})
    if where == "keys":
        assert out[:, 2:].isnan().all() and lse[:, 2:].isnan().all()
    else:
        assert out[:, 2:, 7].isnan().all() and lse.isfinite().all()
        out[:, 2:, 7] = 0
        assert out.isfinite().all()
