"""Single tokens and short chunks over tables with much room: values that are not finite where a row does not look, at places that
leave the keys of one request to several wavefronts and workgroups, each of which does its part again."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import attention_plain as plain  # noqa: E402
from test_gpu_attention import BF, F16, Paged  # noqa: E402

# (requests, heads, tokens): tiles of 16 rows up to three tokens, of 32 for seven; few and many shares in a workgroup
FORMS = [(4, 8, 1), (4, 8, 3), (200, 8, 1), (200, 8, 3), (24, 8, 7), (200, 8, 7)]


def case(dtype, requests, heads, tokens, dim, seed):
    lens = [501 - 7 * (r % 5) for r in range(requests)]
    return lens, Paged(dtype, heads, 2, dim, 16, lens, [tokens] * requests, seed=seed, width=100)


def places(p, lens, first, end):
    """(page, place) of the positions first(n) .. end(n) - 1 of every request of length n."""
    at = [(r, j) for r, n in enumerate(lens) for j in range(max(first(n), 0), end(n))]
    r, j = torch.tensor(at, device="cuda").T
    return p.table[r, j // 16].long(), j % 16


@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("requests,heads,tokens", FORMS)
def test_values_that_have_left_the_window(dtype, dim, requests, heads, tokens):
    lens, p = case(dtype, requests, heads, tokens, dim, 1)
    window = 150
    rows = [0, tokens - 1, requests * tokens // 2, requests * tokens - 1]
    want = p.want(window, rows)
    page, place = places(p, lens, lambda n: 0, lambda n: n - tokens - window + 1)
    p.v[page, place] = torch.where(place % 3 > 0, math.nan, -math.inf).to(dtype)[:, None, None]
    p.k[page, place] = torch.where(place % 2 > 0, math.inf, math.nan).to(dtype)[:, None, None]
    got = p.run(window)
    assert got[0].isfinite().all() and got[1].isfinite().all()
    plain.check(got, want)


@pytest.mark.parametrize("dtype", [BF, F16], ids=["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("requests,heads,tokens", [f for f in FORMS if f[2] > 1])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_a_value_that_only_the_last_token_sees(dtype, dim, requests, heads, tokens, bad):
    lens, p = case(dtype, requests, heads, tokens, dim, 2)
    rows = [0, tokens - 2, requests * tokens - 2]
    want = p.want(0, rows)
    last = [(r + 1) * tokens - 1 for r in range(requests)]
    page, place = places(p, lens, lambda n: n - 1, lambda n: n)
    p.v[page, place, 1, 3] = bad
    out, lse = p.run()
    plain.check((out, lse), want)
    odd = ~out.isfinite()
    assert odd[last, heads // 2:, 3].all() and lse.isfinite().all()
    odd[last, heads // 2:, 3] = False
    assert not odd.any()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("requests,heads,tokens", [f for f in FORMS if f[2] > 1])
def test_a_key_that_only_the_last_token_sees(dim, requests, heads, tokens):
    lens, p = case(BF, requests, heads, tokens, dim, 3)
    rows = [0, tokens - 2, requests * tokens - 2]
    want = p.want(0, rows)
    last = [(r + 1) * tokens - 1 for r in range(requests)]
    page, place = places(p, lens, lambda n: n - 1, lambda n: n)
    p.k[page, place, 1, 3] = math.nan
    out, lse = p.run()
    plain.check((out, lse), want)
    odd = ~out.isfinite()
    assert odd[last, heads // 2:].all() and lse[last, heads // 2:].isnan().all()
    odd[last, heads // 2:] = False
    assert not odd.any()
