"""The calls over 8 bits at their edges: dimensions of one whose strides mean nothing, queries that are not numbers, whole parts of a request that are
not, values hidden from some rows at every place that wavefronts and workgroups share keys, scales next to 0, long tails of small weights, two
streams at once."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2601_07048_amd import jx  # noqa: E402

import attention8_plain as plain8  # noqa: E402
import attention_plain as plain  # noqa: E402
from test_gpu_attention import BF, F16, TYPES, i32, normal  # noqa: E402
from test_gpu_attention8 import CODE, NAN_CODE, NAN_SCALE, SCALE, Paged8, cache8, found8_case  # noqa: E402
from test_gpu_attention_ones import odd  # noqa: E402


# ---- dimensions of one -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("heads,kv,page,block,length", [(4, 1, 16, 8, 100), (1, 1, 1, 1, 20), (3, 1, 64, 64, 64), (1, 1, 16, 2, 16)])
@pytest.mark.parametrize("new", [1, 16])
def test_strides_of_dimensions_of_one(heads, kv, page, block, length, new):
    p = Paged8(BF, heads, kv, 64, page, block, [length], [new], seed=1, spare=0)
    want = p.run()
    p.q, p.k = odd(p.q), odd(p.k)  # the values' strides stay
    got = p.run()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    p.v = odd(p.v)
    got = p.run()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_strides_of_dimensions_of_one_in_a_store_and_a_list():
    q, k, v = (normal((1, 1, 64), BF, i) for i in range(3))
    codes = [torch.zeros((1, 1, 1, 64), dtype=torch.uint8, device="cuda").view(CODE) for _ in range(4)]
    scale = [torch.zeros((1, 1, 1), dtype=torch.uint8, device="cuda").view(SCALE) for _ in range(4)]
    pos, slot = i32([0]), torch.zeros(1, dtype=torch.int64, device="cuda")
    want = jx.qk_norm_rope8(q, k, v, codes[0], codes[1], scale[0], scale[1], pos, slot)
    got = jx.qk_norm_rope8(odd(q), odd(k), odd(v), odd(codes[2]), codes[3], scale[2], scale[3], pos, slot)
    assert torch.equal(got, want)
    for x in (codes, scale):
        assert torch.equal(x[0].view(torch.uint8), x[2].view(torch.uint8)) and torch.equal(x[1].view(torch.uint8), x[3].view(torch.uint8))
    q, keys, values, ks, vs, ids = found8_case(BF, 1, 1, 1, 64, 5, 1, 1, seed=2, holes=0.0)
    want = jx.found_attention8(q, keys, values, ks, vs, ids, 0.1, 1)
    got = jx.found_attention8(odd(q), odd(keys), values, ks, vs, ids, 0.1, 1)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# ---- what is not a number ----------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("new", [1, 3, 40])
@pytest.mark.parametrize("lens", [[60], [250], [3000], [700, 64, 5000, 130]], ids=["unit", "own", "one", "unlike"])
@pytest.mark.parametrize("kv,dim", [(2, 128), (4, 64)])
def test_a_query_that_is_not_a_number(dtype, new, lens, kv, dim):
    p = Paged8(dtype, 4, kv, dim, 16, 16, lens, [min(new, n) for n in lens], seed=new)
    rows = p.q.shape[0]
    bad = sorted({0, rows // 2, rows - 1})
    p.q[bad, 1, 5] = math.nan
    out, lse = p.run()
    assert out[bad, 1].isnan().all() and lse[bad, 1].isnan().all()
    want = p.want(rows=bad)
    plain.check((out, lse), {at: w for at, w in want.items() if at[1] != 1})
    out[bad, 1], lse[bad, 1] = 0, 0
    assert out.isfinite().all() and lse.isfinite().all()


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("new", [1, 3, 40])
@pytest.mark.parametrize("where", ["keys", "values", "keys' scales", "values' scales"])
@pytest.mark.parametrize("length,first", [(250, 64), (3000, 0), (3000, 1984), (3000, 2928), (20000, 6400)])
def test_what_is_not_a_number_over_a_whole_part(dtype, new, where, length, first):
    """Whole units of keys in a row, as many as a part of a request has at the least; all new tokens stand behind them or among them."""
    p = Paged8(dtype, 4, 2, 128, 16, 16, [length], [new], seed=first)
    end = min(first + 64, (length - new + 1) // 16 * 16)  # so that every row sees them, whole blocks
    assert end > first
    for j in range(first, end):
        page, place = p.place(0, j)
        if "scales" in where:
            (p.k_scale if "keys" in where else p.v_scale).view(torch.uint8)[page, place // 16, 1] = NAN_SCALE
        else:
            (p.k if "keys" in where else p.v).view(torch.uint8)[page, place, 1, 7] = NAN_CODE
    out, lse = p.run()
    plain.check((out, lse), {at: w for at, w in p.want(rows=[0, new - 1]).items() if at[1] < 2})
    if "keys" in where:
        assert out[:, 2:].isnan().all() and lse[:, 2:].isnan().all()
        return
    gone = slice(7, 8) if where == "values" else slice(0, 128)
    assert out[:, 2:, gone].isnan().all() and lse.isfinite().all()
    out[:, 2:, gone] = 0
    assert out.isfinite().all()


# (requests, heads, tokens): tiles of 16 rows up to three tokens, of 32 for seven; few and many shares in a workgroup
FORMS = [(4, 8, 1), (4, 8, 3), (200, 8, 1), (200, 8, 3), (24, 8, 7), (200, 8, 7)]


def many(dtype, requests, heads, tokens, dim, block, seed):
    lens = [501 - 7 * (r % 5) for r in range(requests)]
    return lens, Paged8(dtype, heads, 2, dim, 16, block, lens, [tokens] * requests, seed=seed, width=100)


def places(p, lens, first, end):
    """(page, place) of the positions first(n) .. end(n) - 1 of every request of length n."""
    at = [(r, j) for r, n in enumerate(lens) for j in range(max(first(n), 0), end(n))]
    r, j = torch.tensor(at, device="cuda").T
    return p.table[r, j // 16].long(), j % 16


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("requests,heads,tokens", FORMS)
def test_values_that_have_left_the_window(dtype, dim, requests, heads, tokens):
    lens, p = many(dtype, requests, heads, tokens, dim, 4, 1)
    window = 150
    rows = [0, tokens - 1, requests * tokens // 2, requests * tokens - 1]
    want = p.want(window, rows)
    page, place = places(p, lens, lambda n: 0, lambda n: n - tokens - window + 1)
    p.v.view(torch.uint8)[page, place] = NAN_CODE
    p.k.view(torch.uint8)[page, place] = 0xFF
    page, place = places(p, lens, lambda n: 0, lambda n: (n - tokens - window + 1) // 4 * 4)
    p.v_scale.view(torch.uint8)[page, place // 4] = NAN_SCALE
    p.k_scale.view(torch.uint8)[page, place // 4] = NAN_SCALE
    got = p.run(window)
    assert got[0].isfinite().all() and got[1].isfinite().all()
    plain.check(got, want)


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("requests,heads,tokens", [f for f in FORMS if f[2] > 1])
@pytest.mark.parametrize("what", ["value", "value's scale", "key"])
def test_what_only_the_last_token_sees(dtype, dim, requests, heads, tokens, what):
    lens, p = many(dtype, requests, heads, tokens, dim, 1, 2)
    rows = [0, tokens - 2, requests * tokens - 2]
    want = p.want(0, rows)
    last = [(r + 1) * tokens - 1 for r in range(requests)]
    page, place = places(p, lens, lambda n: n - 1, lambda n: n)
    if what == "value's scale":
        p.v_scale.view(torch.uint8)[page, place, 1] = NAN_SCALE
    else:
        (p.v if what == "value" else p.k).view(torch.uint8)[page, place, 1, 3] = NAN_CODE
    out, lse = p.run()
    plain.check((out, lse), want)
    gone = ~out.isfinite()
    if what == "value":
        assert gone[last, heads // 2:, 3].all()
        gone[last, heads // 2:, 3] = False
    else:
        assert gone[last, heads // 2:].all()
        gone[last, heads // 2:] = False
    assert not gone.any()
    if what == "key":
        assert lse[last, heads // 2:].isnan().all()
    else:
        assert lse.isfinite().all()


# ---- scores and weights ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("lens", [[200], [3000]])
@pytest.mark.parametrize("scale,size", [(0.0, 46), (-0.0, 49), (1e-33, 53), (-2e-37, 56), (1e-30, 46)])
def test_small_scales_of_large_products(new, lens, scale, size):
    """Queries and keys 2^size times as large.  Products of up to 375 times that twice (in 64 bits), 2^120.6: float32 has to hold them, which it does not
    from 2^60 on, where one of these comes to 5.0e38."""
    p = Paged8(BF, 4, 2, 64, 16, 8, lens, [new], seed=3)
    p.q = (p.q.float() * 2.0 ** size).to(BF)
    byte = p.k_scale.view(torch.uint8)
    byte[byte != NAN_SCALE] += size
    p.scale = scale
    p.check(rows=[0, new - 1])


@pytest.mark.parametrize("below", [12.0, 18.0, 21.0], ids=lambda x: f"{x:.0f} nats")
@pytest.mark.parametrize("tokens,page", [(1, 16), (3, 16), (3, 8)], ids=["16 rows", "32 rows", "128 rows"])
@pytest.mark.parametrize("dim", [64, 128])
def test_a_long_tail_counts(below, tokens, page, dim):
    """binary16: one key with nearly all the weight, and many others that each have next to none but count together.  Weights are rounded 2^7 times as
    large as they are beside the running maximum, so that half the type's smallest step, 2^-25, is 2^-32 of the largest weight: n keys add at most
    2^-32 sum_j |v_j|, in place of tiny / 2 sum_j |v_j| among the bounds of attention_plain.  Of more than 1,024 requests each one's keys are taken in one
    go, so that all of the tail stands beside the first key."""
    n, others = 60000, 1030
    p = Paged8(F16, 8, 1, dim, page, 8, [n] + [4] * others, [tokens] * (1 + others), seed=dim, spare=0)
    p.scale = 1.0
    at = p.table[0, :n // page].long()
    k, v = (x.view(torch.uint8)[at].flatten(0, 1).clone().view(CODE).float() * s.view(torch.uint8)[at].flatten(0, 1).clone().view(SCALE).float().repeat_interleave(8, 0)[..., None]
            for x, s in ((p.k, p.k_scale), (p.v, p.v_scale)))
    k[:, 0, 0] = -below
    k[0] = 0
    v.abs_()
    v[0] = 0
    held = []
    for x, codes, scale in ((k, p.k, p.k_scale), (v, p.v, p.v_scale)):
        c, s = plain8.quantised(x.cpu(), 8)
        codes.view(torch.uint8)[at] = c.view(torch.uint8).unflatten(0, (-1, page)).cuda()
        scale.view(torch.uint8)[at] = s.view(torch.uint8).unflatten(0, (-1, page // 8)).cuda()
        held.append(plain8.rows_stand_for(c, s, 8)[:, 0])
    p.q.mul_(0.02)
    p.q[:tokens, :, 0] = 1
    out, lse = p.run()
    k, v = held
    for t in range(tokens):
        seen = n - tokens + 1 + t
        for h in (0, 5):
            q = p.q[t, h].cpu().double()
            o, l, bo, bl = plain.attend_row(q, k[:seen], v[:seen], 1.0, F16, rounded=False)
            w = torch.exp(k[:seen] @ q - l)
            bo = bo + (plain.UNIT[F16] * (w @ v[:seen]) + 2.0 ** -32 * v[:seen].sum(0)) * 1.02
            err = (out[t, h].cpu().double() - o).abs()
            assert bool((err <= bo).all()), (t, h, float((err / o).max()))
            assert abs(float(lse[t, h]) - l) <= bl
    assert out.isfinite().all() and math.isfinite(float(lse.sum()))


@pytest.mark.parametrize("tokens,page", [(1, 16), (3, 16), (3, 8)], ids=["16 rows", "32 rows", "128 rows"])
def test_weights_at_the_top_of_their_range(tokens, page):
    """Scores that rise by just under 2^8 over the running maximum, which then stays: weights of up to 2^15 times values near binary16's largest, and sums
    of them, stay numbers."""
    n = 400
    p = Paged8(F16, 8, 1, 64, page, 8, [n] + [4] * 1030, [tokens] * 1031, seed=1, spare=0)
    at = p.table[0, :n // page].long()
    k = torch.zeros((n, 1, 64))
    k[64:, 0, 0] = 5.5  # 7.93 times log 2
    for x, codes, scale in ((k, p.k, p.k_scale), (torch.full((n, 1, 64), 61440.0), p.v, p.v_scale)):
        c, s = plain8.quantised(x, 8)
        assert bool((plain8.rows_stand_for(c, s, 8) == x).all())
        codes.view(torch.uint8)[at] = c.view(torch.uint8).unflatten(0, (-1, page)).cuda()
        scale.view(torch.uint8)[at] = s.view(torch.uint8).unflatten(0, (-1, page // 8)).cuda()
    p.q.zero_()
    p.q[:tokens, :, 0] = 1
    p.scale = 1.0
    p.check(rows=list(range(tokens)))


# ---- the store ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("t", [3, 6000])
@pytest.mark.parametrize("dim,rot", [(64, 32), (64, 0), (128, 16)])
@pytest.mark.parametrize("pairs", [False, True])
def test_infinities_behind_the_turned_elements(dtype, t, dim, rot, pairs):
    """Queries keep them; a key's is held as what is not a number, and the others of its block are what they are without it."""
    heads, kv, block = 8, 2, 8
    q, k, v = normal((t, heads, dim), dtype, 1), normal((t, kv, dim), dtype, 2), normal((t, kv, dim), dtype, 3)
    q[:, 1, rot + 3], q[:, 2, dim - 1] = math.inf, -math.inf
    angle = torch.rand((t, rot // 2), generator=torch.Generator().manual_seed(4)).cuda()
    cos, sin = (angle.cos(), angle.sin()) if rot else (None, None)
    slot = torch.arange(t, device="cuda")
    end = []
    for bad in (0.0, math.inf):
        k[:, 1, rot + 9] = bad
        (kc, ks), (vc, vs) = (cache8(t // 16 + 1, 16, kv, dim, block, i) for i in (1, 2))
        got = jx.qk_norm_rope8(q, k, v, kc, vc, ks, vs, i32(list(range(t))), slot, cos, sin, interleaved=pairs)
        assert torch.equal(got[:, :, rot:], q[:, :, rot:]) and got[:, :, :rot].isfinite().all()
        end.append([x.view(torch.uint8).clone() for x in (kc, ks, vc, vs)])
    codes = [x[0].flatten(0, 1)[:t] for x in end]
    assert ((codes[1][:, 1, rot + 9] & 0x7F) == NAN_CODE).all()
    for x in codes:
        x[:, 1, rot + 9] = 0
    assert torch.equal(codes[0], codes[1]) and all(torch.equal(x, y) for x, y in zip(end[0][1:], end[1][1:]))


# ---- two streams -------------------------------------------------------------------------------------------------------

def test_calls_on_two_streams_at_once():
    """Store, attention and found rows of two programs side by side, each with tensors of its own: what each gives is what it gives alone."""
    def program(seed):
        p = Paged8(BF, 16, 4, 128, 16, 16, [3000, 17, 900, 2500], [1, 1, 33, 1] if seed else [1, 1, 1, 1], seed=seed)
        t = p.q.shape[0]
        q, keys, values, ks, vs, ids = found8_case(BF, t, 16, 4, 128, 50, 400, 16, seed=seed)
        k, v = normal((t, 4, 128), BF, seed + 1), normal((t, 4, 128), BF, seed + 2)
        at = torch.arange(t, device="cuda")
        caches = [x for i in (5, 6) for x in cache8(4, 16, 4, 128, 16, seed + i)]

        def step():
            ready = jx.qk_norm_rope8(q, k, v, caches[0], caches[2], caches[1], caches[3], at.int(), at)
            part = jx.paged_attention8(p.q, p.k, p.v, p.k_scale, p.v_scale, p.table, p.q_start, p.kv_len, p.scale)
            out = jx.found_attention8(ready, keys, values, ks, vs, ids, p.scale, 16, part=part)
            return [ready, *part, *out, *(x.view(torch.uint8).clone() for x in caches)]
        return step

    steps = [program(0), program(7)]
    want = [s() for s in steps]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in steps]
    got = [[], []]
    for _ in range(8):
        for i, (s, stream) in enumerate(zip(steps, streams)):
            with torch.cuda.stream(stream):
                got[i].append(s())
    torch.cuda.synchronize()
    for w, runs in zip(want, got):
        for run in runs:
            assert all(torch.equal(x, y) for x, y in zip(run, w))
