"""Attention beside the index against its definitions in 64 bits: paged attention over all that a table, a window and a chunk can
leave of the keys, attention over found rows and its join, norm, rotation and store, and the cache's bookkeeping.  The bounds are
those of attention_plain."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2601_07048_amd import jx  # noqa: E402

import attention_plain as plain  # noqa: E402

TYPES = [torch.bfloat16, torch.float16]
BF, F16 = TYPES


def normal(shape, dtype, seed, gain=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * gain).to(dtype).cuda()


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda").contiguous()


class Paged:
    """Requests with lengths `lens` (new tokens included) of which the last `new` ask; pages scattered, what no request owns is NaN."""

    def __init__(self, dtype, heads, kv, dim, page, lens, new, seed=0, layout="thd", spare=3, width=None, pad=0):
        rng = np.random.default_rng(seed)
        held = [-(-max(n, 0) // page) for n in lens]
        pages = sum(held) + spare
        order = rng.permutation(pages)
        width = width or max(1, max(held) + 1)
        table = np.full((len(lens), width), -1, np.int32)
        at = 0
        for r, n in enumerate(held):
            m = min(n, width)
            table[r, :m] = order[at:at + m]
            at += n
        shape = {"thd": (pages, page, kv, dim), "htd": (pages, kv, page, dim)}[layout]
        k, v = normal(shape, dtype, seed + 1), normal(shape, dtype, seed + 2)
        if layout == "htd":
            k, v = k.transpose(1, 2), v.transpose(1, 2)
        free = torch.ones((pages, page), dtype=torch.bool, device="cuda")
        for r, n in enumerate(lens):
            for p in range(min(held[r], width)):
                free[int(table[r, p]), :min(page, n - p * page)] = False
        k[free], v[free] = math.nan, math.nan
        self.k, self.v, self.table = k, v, i32(table)
        self.q_start = i32(np.cumsum([0] + list(new)).tolist())
        self.kv_len = i32(list(lens))
        self.q = normal((sum(new) + pad, heads, dim), dtype, seed + 3, 1.5)
        self.scale = dim ** -0.5

    def run(self, window=0, **kw):
        got = jx.paged_attention(self.q, self.k, self.v, self.table, self.q_start, self.kv_len, self.scale, window=window, **kw)
        torch.cuda.synchronize()
        return got

    def want(self, window=0, rows=None):
        return plain.paged(self.q, self.k, self.v, self.table, self.q_start, self.kv_len, self.scale, window, rows)

    def check(self, window=0, rows=None, what=""):
        got = self.run(window)
        assert torch.isfinite(got[0]).all(), what
        plain.check(got, self.want(window, rows), what)
        return got


# ---- paged attention ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("heads,kv,dim,page", [(8, 1, 128, 16), (6, 2, 64, 8), (4, 4, 96, 32), (5, 1, 256, 64), (3, 3, 8, 1), (16, 1, 80, 4),
                                               (40, 2, 128, 128), (2, 1, 192, 16), (33, 1, 64, 2)])
def test_one_token_per_request(dtype, heads, kv, dim, page):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 127, 130, 257]
    Paged(dtype, heads, kv, dim, page, lens, [1] * len(lens), seed=dim + heads).check()


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("heads,kv,dim,page", [(8, 2, 128, 16), (4, 4, 64, 64), (7, 1, 128, 8), (4, 2, 256, 32), (2, 2, 72, 16), (12, 2, 96, 1)])
@pytest.mark.parametrize("window", [0, 1, 5, 64, 1000])
def test_chunks_of_unlike_lengths(dtype, heads, kv, dim, page, window):
    lens, new = [70, 1, 33, 129, 5, 64, 200], [70, 1, 17, 3, 0, 64, 65]
    Paged(dtype, heads, kv, dim, page, lens, new, seed=window).check(window)


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("new", [[1], [2], [16], [17], [100], [300]], ids=lambda n: str(n[0]))
def test_one_request(dtype, new):
    Paged(dtype, 4, 1, 128, 16, [333], new, seed=new[0]).check()


def test_no_keys_no_requests_and_rows_of_none():
    # lengths of zero, fewer tokens in the cache than ask, rows before the first and after the last request
    p = Paged(BF, 4, 2, 64, 16, [0, 3, 40, 0], [2, 5, 0, 0], seed=5, pad=3)
    got = p.check()
    assert (got[1][:4] == -math.inf).all() and (got[1][4:7] > -math.inf).all() and (got[1][7:] == -math.inf).all()
    p.q_start += 2
    p.check()
    p.q_start = i32([0])
    p.kv_len, p.table = i32([]), p.table[:0].contiguous()
    out, lse = p.run()
    assert not out.any() and (lse == -math.inf).all()
    p.q = p.q[:0]
    assert p.run()[0].shape[0] == 0


@pytest.mark.parametrize("new", [1, 50])
def test_pages_that_the_table_does_not_name(new):
    p = Paged(F16, 8, 2, 128, 16, [150, 150, 150, 150], [new] * 4, seed=9)
    pages = p.k.shape[0]
    p.table[0, 2] = -1
    p.table[1, :5] = -1
    p.table[2, 9] = pages        # names no page
    p.table[2, 3] = 2 ** 31 - 1
    p.table[3] = -7              # nothing is left
    got = p.check()
    assert (got[1][3 * new:] == -math.inf).all()
    p.check(window=40)
    p.table = p.table[:, :6].contiguous()  # a table narrower than the lengths
    p.check()


@pytest.mark.parametrize("heads,kv,dim", [(8, 2, 128), (2, 2, 64), (4, 1, 256)])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_what_a_row_does_not_see_has_no_part_in_it(heads, kv, dim, bad):
    """A key or value that is not a number, at every place of a chunk in turn: the rows before it, and those that their window has
    taken past it, are what they are without it."""
    for at in (10, 11, 40, 63, 64, 88, 89):
        p = Paged(BF, heads, kv, dim, 16, [90], [80], seed=at)
        row = at - 10  # the row at that position
        before = list(range(max(0, row - 3), row))
        past = [r for r in range(row + 7, min(80, row + 10))]
        want, want_window = p.want(rows=before), p.want(window=7, rows=before + past)
        page, place = int(p.table[0, at // 16]), at % 16
        for cache in (p.k, p.v):
            keep = cache[page, place].clone()
            cache[page, place] = bad
            got = p.run()
            assert torch.isfinite(got[0][:row]).all() and torch.isfinite(got[1][:row]).all()
            plain.check(got, want, (at, "chunk"))
            if cache is p.v:
                assert not torch.isfinite(got[0][row:]).any()
            got = p.run(window=7)
            assert torch.isfinite(got[0][:row]).all() and torch.isfinite(got[0][row + 7:]).all()
            plain.check(got, want_window, (at, "window"))
            cache[page, place] = keep


@pytest.mark.parametrize("heads,kv", [(1, 1), (8, 2), (40, 2)])
@pytest.mark.parametrize("dim", [64, 128, 200])
def test_single_tokens_do_not_see_what_has_left_their_window(heads, kv, dim):
    """Before the window, behind the length and in pages that the table does not name there may be anything."""
    p = Paged(BF, heads, kv, dim, 16, [150, 75, 33, 16], [1] * 4, seed=dim)
    want = p.want(window=20)
    for r, n in enumerate((150, 75, 33, 16)):
        for j in range(n - 20):
            page, place = int(p.table[r, j // 16]), j % 16
            p.k[page, place] = math.inf if j % 2 else math.nan
            p.v[page, place] = math.nan if j % 3 else -math.inf
    plain.check(p.run(window=20), want)


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
def test_values_that_are_infinite_reach_the_rows_that_see_them(dtype):
    p = Paged(dtype, 4, 2, 64, 16, [50], [20], seed=4)
    p.v[int(p.table[0, 2]), 8, 1, 3] = math.inf  # position 40 = row 10, key head 1
    got = p.run()
    assert (got[0][10:, 2:, 3] == math.inf).all() and torch.isfinite(got[0][:10]).all() and torch.isfinite(got[0][:, :2]).all()
    assert torch.isfinite(got[0][10:, 2:, :3]).all() and torch.isfinite(got[0][10:, 2:, 4:]).all()


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
def test_scores_of_every_size(dtype):
    """Scores from -3e4 to 3e4: the largest one decides, nothing overflows; and equal scores, where the mean is the result."""
    p = Paged(dtype, 8, 2, 128, 16, [777, 400], [1, 130], seed=3)
    p.q *= 100
    p.scale = 2.0
    p.check(rows=[0, 1, 50, 130])
    p.q.zero_()
    p.check(rows=[0, 1, 130])
    p.scale = -0.1
    p.q = normal(p.q.shape, dtype, 1)
    p.check(rows=[0, 1, 130])
    # every score below the type's lowest value: rising along the keys, so that each tile brings a new largest one
    ramp = torch.arange(777, device="cuda").float()
    for j in range(777):
        p.k[int(p.table[0, j // 16]), j % 16] = (-(777 - ramp[j]) / 8).to(dtype)
    p.q[0] = 8.0
    p.scale = 1.0
    p.check(rows=[0])


@pytest.mark.parametrize("layout", ["thd", "htd"])
def test_strides(layout):
    p = Paged(BF, 8, 2, 64, 16, [100, 37], [1, 20], seed=8, layout=layout)
    want = p.run()
    fused = torch.full((21, 12, 80), math.nan, dtype=BF, device="cuda")
    fused[:, 2:10, :64] = p.q
    q = p.q
    p.q = fused[:, 2:10, :64]
    assert torch.equal(p.run()[0], want[0])
    p.q = q
    pages = p.k.shape[0]  # keys and values of a page together, one block for both
    both = torch.full((pages, 2, 16, 3, 72), math.nan, dtype=BF, device="cuda")
    both[:, 0, :, 1:, :64], both[:, 1, :, 1:, :64] = p.k, p.v
    p.k, p.v = both[:, 0, :, 1:, :64], both[:, 1, :, 1:, :64]
    assert torch.equal(p.run()[0], want[0])
    p.check()
    assert torch.equal(p.run(out=(torch.empty_like(want[0]), None))[0], want[0])


def test_offsets_beyond_32_bits():
    stride = 2 ** 31 + 2 ** 20  # elements between pages
    pool = torch.empty(2 * stride + 2 * 64 * 2 * 64, dtype=BF, device="cuda")
    k = pool.as_strided((3, 64, 2, 64), (stride, 128, 64, 1), 0)
    v = pool.as_strided((3, 64, 2, 64), (stride, 128, 64, 1), 64 * 128)
    for new in (1, 30):
        p = Paged(BF, 4, 2, 64, 64, [170], [new], seed=2, spare=0)
        want = p.run()
        k.copy_(p.k)
        v.copy_(p.v)
        p.k, p.v = k, v
        assert torch.equal(p.run()[0], want[0])
        p.check(rows=[0])


@pytest.mark.parametrize("new", [1, 3, 40])
@pytest.mark.parametrize("lens", [[20011], [5, 9000, 1, 700, 4096], [2000] * 40], ids=["one", "unlike", "many"])
def test_long_caches(lens, new):
    lens = [max(n, 1) for n in lens]
    p = Paged(BF, 16, 2, 128, 16, lens, [min(new, n) for n in lens], seed=len(lens))
    rows = sorted({0, p.q.shape[0] // 2, p.q.shape[0] - 1})
    p.check(rows=rows)
    p.check(window=777, rows=rows)


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 72, 96, 128, 192, 256])
@pytest.mark.parametrize("window", [0, 30])
def test_a_few_tokens_of_short_requests(dtype, dim, window):
    rng = np.random.default_rng(dim)
    lens = rng.integers(1, 140, 24).tolist()
    new = [min(int(rng.integers(1, 9)), n) for n in lens]
    Paged(dtype, 8, 2, dim, 16, lens, new, seed=dim).check(window, rows=list(range(0, sum(new), 3)))


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("bad", [None, math.nan])
def test_short_requests_in_narrow_and_wide_tables(dtype, dim, bad):
    """How much a table has room for decides who takes the keys, and nothing else; the same for a window that is short."""
    lens = [0, 1, 3, 64, 65, 100, 127, 128]
    p = Paged(dtype, 8, 2, dim, 16, lens, [1, 1, 1, 2, 1, 1, 2, 1], seed=dim, width=8)
    if bad is not None:  # the first key of the request of 64: its rows 3 and 4 see it, unless the window is short
        p.v[int(p.table[3, 0]), 0, 1, 3] = bad
    rows = [t for t in range(10) if bad is None or t not in (3, 4)]
    narrow, short = p.run(), p.run(window=40)
    p.table = torch.cat([p.table, torch.full((len(lens), 200), -1, dtype=torch.int32, device="cuda")], 1)
    for what, got, window in (("narrow", narrow, 0), ("wide", p.run(), 0), ("narrow, window", short, 40), ("wide, window", p.run(window=40), 40)):
        plain.check(got, p.want(window, None if window else rows), what)
        for t in range(10):
            if t not in rows and not window:
                o = got[0][t].isfinite()
                assert not o[4:, 3].any() and o[:4].all() and o[4:, :3].all() and o[4:, 4:].all(), what


@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("lens,new", [([700], [600]), ([1500, 1100], [1100, 1100]), ([90, 3000], [1, 2100])], ids=["one", "two", "unlike"])
def test_long_chunks(dim, lens, new):
    p = Paged(BF, 8, 2, dim, 32, lens, new, seed=dim)
    rows = sorted({0, 1, 63, 64, 127, 128, 255, 256, sum(new) // 2, sum(new) - 1})
    p.check(rows=rows)
    p.check(window=100, rows=rows)


def test_more_tiles_than_are_shared_out():
    """Many rows: each tile is a workgroup's, none is joined."""
    rng = np.random.default_rng(3)
    lens = rng.integers(6, 80, 1100).tolist()
    p = Paged(BF, 8, 1, 64, 4, lens, [6] * 1100, seed=2)
    p.check(rows=list(range(0, 6600, 371)))
    p.check(window=9, rows=list(range(5, 6600, 371)))


def test_a_scale_of_zero_gives_the_mean():
    for new in (1, 40):
        p = Paged(F16, 4, 2, 64, 16, [100, 41], [new, new], seed=4)
        p.scale = 0.0
        p.check()


def test_many_requests():
    rng = np.random.default_rng(0)
    lens = rng.integers(0, 90, 1500).tolist()
    new = [int(rng.integers(0, 3)) for _ in lens]
    p = Paged(F16, 4, 1, 64, 16, lens, new, seed=1)
    got = p.check(rows=list(range(0, sum(new), 37)))
    assert torch.isfinite(got[0]).all()


def test_same_bits_every_time_and_on_another_stream():
    p = Paged(BF, 8, 1, 128, 16, [3000, 17, 900], [1, 1, 33], seed=6)
    want = p.run()
    for _ in range(3):
        got = p.run()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = jx.paged_attention(p.q, p.k, p.v, p.table, p.q_start, p.kv_len, p.scale)
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# ---- attention over found rows -----------------------------------------------------------------------------------------

def found_case(dtype, t, heads, kv, dim, k, rows, seed, holes=0.2):
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, rows, (t, heads, k), generator=g, dtype=torch.int32)
    ids[torch.rand((t, heads, k), generator=g) < holes] = -1
    return (normal((t, heads, dim), dtype, seed + 1, 1.5), normal((rows, kv, dim), dtype, seed + 2), normal((rows, kv, dim), dtype, seed + 3),
            ids.cuda())


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("t,heads,kv,dim,k", [(1, 1, 1, 128, 1), (3, 8, 2, 128, 10), (5, 6, 3, 64, 33), (2, 4, 1, 256, 100), (2, 2, 2, 80, 7),
                                              (1, 4, 4, 8, 130), (2, 3, 1, 192, 64), (7, 2, 1, 128, 513)])
@pytest.mark.parametrize("joined", [False, True])
def test_found_rows(dtype, t, heads, kv, dim, k, joined):
    q, keys, values, ids = found_case(dtype, t, heads, kv, dim, k, 50, seed=k)
    ids[0, 0, 0] = 50              # outside
    ids[-1, -1] = -1               # nothing found
    ids[0, -1, :2] = 3             # the same row twice
    part = None
    if joined:
        part = normal((t, heads, dim), dtype, 9), torch.randn((t, heads), generator=torch.Generator().manual_seed(1)).cuda() * 3
        part[1][0, 0] = -math.inf  # a part of no keys, whatever its rows hold
        part[0][0, 0] = math.nan
    scale = dim ** -0.5
    got = jx.found_attention(q, keys, values, ids, scale, part=part)
    torch.cuda.synchronize()
    plain.check(got, plain.found(q, keys, values, ids, scale, part))
    if joined:  # in place
        same = jx.found_attention(q, keys, values, ids, scale, part=part, out=part)
        assert torch.equal(same[0], got[0]) and torch.equal(same[1], got[1])


def test_found_rows_of_no_list_and_rows_that_are_passed_over():
    q, keys, values, ids = found_case(BF, 3, 4, 2, 64, 8, 20, seed=3, holes=0.0)
    out, lse = jx.found_attention(q, keys, values, ids[:, :, :0].contiguous(), 0.1)
    assert not out.any() and (lse == -math.inf).all()
    ids[ids == 7] = 8
    want = jx.found_attention(q, keys, values, ids, 0.1)
    keys[7], values[7] = math.nan, math.inf
    ids[:, :, 3] = -1
    clean = jx.found_attention(q, keys, values, ids, 0.1)
    assert torch.isfinite(clean[0]).all() and not torch.equal(clean[0], want[0])
    # strided rows: only some of a larger table, keys and values of a row together
    both = torch.full((20, 2, 3, 72), math.nan, dtype=BF, device="cuda")
    both[:, 0, :2, :64], both[:, 1, :2, :64] = keys, values
    got = jx.found_attention(q, both[:, 0, :2, :64], both[:, 1, :2, :64], ids, 0.1)
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])


def test_parts_join_to_the_whole():
    """Paged attention over one half of the keys and found attention over the other = attention over all."""
    p = Paged(F16, 8, 2, 128, 16, [64], [4], seed=11)
    whole = p.want()
    k, v = p.k[p.table[0, :4].long()].flatten(0, 1), p.v[p.table[0, :4].long()].flatten(0, 1)
    p.table[0, :2] = -1
    part = p.run()
    ids = torch.arange(32, device="cuda", dtype=torch.int32).expand(4, 8, 32).contiguous()
    got = jx.found_attention(p.q, k[:32], v[:32], ids, p.scale, part=part)
    out = got[0].cpu().double()
    for (t, h), (o, l, bo, bl) in whole.items():
        # the part was rounded to the element type once more
        assert bool(((out[t, h] - o).abs() <= bo + 2 * plain.UNIT[F16] * v.abs().max().cpu().double()).all())
        assert abs(float(got[1][t, h]) - l) <= 4 * bl


# ---- norm, rotation, store ---------------------------------------------------------------------------------------------

def rope_plain(x, weight, eps, cos, sin, pairs):
    """(y, bound without the final rounding) in 64 bits.  The mean square: dim + 8 roundings of float32, square root and divisions
    one each, so the norm is within (dim + 8) 2^-24, the turned pair within 4 more of |a| + |b|."""
    x = x.double().clone()
    dim = x.shape[-1]
    if weight is not None:
        x = x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * weight.double()
    rot = 2 * cos.shape[-1] if cos is not None else 0
    size = x.abs()
    if rot:
        c, s = cos.double()[:, None], sin.double()[:, None]
        lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if pairs else (slice(0, rot // 2), slice(rot // 2, rot))
        a, b = x[..., lo].clone(), x[..., hi].clone()
        x[..., lo], x[..., hi] = a * c - b * s, b * c + a * s
        size[..., lo] = size[..., hi] = a.abs() + b.abs()
    return x, size * (dim + 16) * 2.0 ** -24


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("t,heads,kv,dim,rot,page", [(1, 8, 2, 128, 128, 16), (37, 6, 3, 64, 32, 8), (9, 4, 1, 96, 96, 32), (5, 2, 2, 256, 64, 64),
                                                     (3, 1, 1, 8, 0, 1), (130, 3, 1, 192, 16, 16), (4, 5, 5, 80, 80, 4), (300, 40, 8, 128, 64, 16)])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("normed", [False, True])
def test_norm_rotation_and_store(dtype, t, heads, kv, dim, rot, page, pairs, normed):
    g = torch.Generator().manual_seed(t)
    fused = normal((t, heads + 2 * kv, dim), dtype, t, 3.0)
    fused[0, 0] = 0  # a row of nothing
    q, k, v = fused.split([heads, kv, kv], 1)
    pages = t // page + 2
    cache = normal((2, pages, page, kv, dim), dtype, 5)
    before = cache.clone()
    n_pos = 700
    pos = torch.randint(0, n_pos, (t,), generator=g, dtype=torch.int32)
    slot = torch.randperm(pages * page, generator=g)[:t]
    if t > 4:
        pos[1], pos[2], slot[3], slot[4] = -1, n_pos, -1, pages * page
    angle = torch.rand((n_pos, rot // 2), generator=g) * 6.3
    cos, sin = (angle.cos().cuda(), angle.sin().cuda()) if rot else (None, None)
    wq, wk = (normal((dim,), dtype, 6), normal((dim,), dtype, 7)) if normed else (None, None)
    got = jx.qk_norm_rope(q, k, v, cache[0], cache[1], pos.cuda(), slot.cuda(), cos, sin, wq, wk, eps=1e-5, interleaved=pairs)
    torch.cuda.synchronize()
    at = pos.long().clamp(0, n_pos - 1)
    turn = (cos.cpu()[at], sin.cpu()[at]) if rot else (None, None)
    here = (pos >= 0) & (pos < n_pos) if rot else pos >= 0
    u, tiny = plain.UNIT[dtype], plain.TINY[dtype]

    def close(a, b, bound):
        assert bool(((a.cpu().double() - b).abs() <= (bound + u * b.abs()) * 1.01 + tiny / 2).all())

    y, bound = rope_plain(q.cpu(), wq.cpu() if normed else None, 1e-5, *turn, pairs)
    close(got[here], y[here], bound[here])
    assert not got[~here].any()
    stored = here & (slot >= 0) & (slot < pages * page)
    y, bound = rope_plain(k.cpu(), wk.cpu() if normed else None, 1e-5, *turn, pairs)
    flat = cache.flatten(1, 2)
    close(flat[0][slot[stored]], y[stored], bound[stored])
    assert torch.equal(flat[1][slot[stored]], v[stored.cuda()])
    others = torch.ones(pages * page, dtype=torch.bool)
    others[slot[stored]] = False
    assert torch.equal(flat[:, others], before.flatten(1, 2)[:, others])


def test_queries_in_place_and_other_cache_orders():
    t, heads, kv, dim = 50, 8, 2, 64
    q, k, v = normal((t, heads, dim), BF, 1), normal((t, kv, dim), BF, 2), normal((t, kv, dim), BF, 3)
    angle = torch.rand((100, 32)) * 6
    cos, sin = angle.cos().cuda(), angle.sin().cuda()
    pos, slot = i32(list(range(t))), torch.arange(t, device="cuda") * 2
    a = torch.zeros((2, 8, 16, kv, dim), dtype=BF, device="cuda")
    b = torch.zeros((2, 8, kv, 16, dim), dtype=BF, device="cuda").transpose(2, 3)
    w = normal((dim,), BF, 4)
    want = jx.qk_norm_rope(q, k, v, a[0], a[1], pos, slot, cos, sin, w, w)
    got = jx.qk_norm_rope(q, k, v, b[0], b[1], pos, slot, cos, sin, w, w, out=q)
    assert got is q and torch.equal(got, want) and torch.equal(a, b)


# ---- the cache's bookkeeping -------------------------------------------------------------------------------------------

def plan_plain(lens, new, table, free, n_free, page, n_tokens, n_pages):
    table = table.copy()
    q_start, kv_len, asked, left, total = [0], [], 0, n_free, 0
    pos, slot = np.full(n_tokens, -1, np.int32), np.full(n_tokens, -1, np.int64)
    for r, (a, n) in enumerate(zip(lens, new)):
        a, n = max(a, 0), max(n, 0)
        first, end = -(-a // page), -(-(a + n) // page)
        begin, total = total, total + n
        asked += end - first
        if end > table.shape[1] or total > n_tokens or (end > first and asked > n_free):
            kv_len.append(0)
        else:
            for i in range(first, end):
                table[r, i] = free[n_free - 1 - (asked - end + i)]
            left -= end - first
            kv_len.append(a + n)
            for i in range(n):
                pos[begin + i] = a + i
                at = table[r, (a + i) // page]
                if 0 <= at < n_pages:
                    slot[begin + i] = int(at) * page + (a + i) % page
        q_start.append(min(total, n_tokens))
    return table, q_start, kv_len, pos, slot, left


@pytest.mark.parametrize("n_req,page,longest,chunk", [(1, 16, 40, 1), (1, 1, 5, 7), (5, 8, 100, 30), (64, 16, 3000, 1), (300, 4, 50, 9), (1025, 32, 200, 40),
                                                      (3000, 16, 20, 2), (8192, 16, 40, 1)])
@pytest.mark.parametrize("slack", [1.5, 1.0, 0.6, 0.0])
def test_plan(n_req, page, longest, chunk, slack):
    rng = np.random.default_rng(n_req)
    lens, new = rng.integers(0, longest, n_req), rng.integers(0, chunk + 1, n_req)
    if n_req > 4:
        lens[1], new[2], new[3] = -5, -3, 0
    la, na = np.maximum(lens, 0), np.maximum(new, 0)
    need = int((-(-(la + na) // page) - -(-la // page)).sum())
    n_pages, width = need * 2 + 5, -(-(longest + chunk) // page)
    table = rng.integers(-1, n_pages + 1, (n_req, width)).astype(np.int32)
    free = rng.permutation(n_pages).astype(np.int32)
    n_free = int(need * slack)
    extra = int(slack * 10) - 8
    n_tokens = max(int(na.sum()) + extra, 0)
    want = plan_plain(lens.tolist(), new.tolist(), table, free, n_free, page, n_tokens, n_pages)
    dt, nf = i32(table), i32([n_free])
    got = jx.kv_plan(i32(lens), i32(new), dt, i32(free), nf, page, n_tokens)
    assert np.array_equal(dt.cpu().numpy(), want[0])
    assert got.q_start.tolist() == want[1] and got.kv_len.tolist() == want[2]
    assert np.array_equal(got.pos.cpu().numpy(), want[3]) and np.array_equal(got.slot.cpu().numpy(), want[4])
    assert int(got.n_free) == want[5] and int(nf) == n_free


def test_plan_limits():
    big = 2 ** 31 - 1
    table = i32(np.full((4, 8), -1))
    free = i32(np.arange(40))
    # sums and lengths that pass 32 bits; a request wider than the table; one that fits
    got = jx.kv_plan(i32([big, 0, 100, 0]), i32([big, big, 29, 0]), table, free, i32([40]), 16, 64)
    assert got.kv_len.tolist() == [0, 0, 0, 0] and got.q_start.tolist() == [0, 64, 64, 64, 64] and int(got.n_free) == 40
    assert (table == -1).all() and (got.slot == -1).all() and (got.pos == -1).all()
    # no requests, no tokens; a count of free pages that is out of range
    got = jx.kv_plan(i32([]), i32([]), table[:0], free, i32([5]), 16, 3)
    assert got.q_start.tolist() == [0] and got.pos.tolist() == [-1] * 3 and int(got.n_free) == 5
    got = jx.kv_plan(i32([3]), i32([0]), table[:1].contiguous(), free, i32([-4]), 16, 0)
    assert got.kv_len.tolist() == [3] and int(got.n_free) == 0
    got = jx.kv_plan(i32([0]), i32([1]), table[:1].contiguous(), free, i32([1000]), 16, 1)
    assert got.slot.tolist() == [39 * 16] and int(got.n_free) == 39


@pytest.mark.parametrize("n_req", [1, 7, 100, 2500])
def test_release(n_req):
    rng = np.random.default_rng(n_req)
    width = 150 if n_req < 1000 else 5
    n_pages = n_req * width + 9
    table = rng.permutation(n_pages)[:n_req * width].reshape(n_req, width).astype(np.int32)
    table[rng.random(table.shape) < 0.3] = -1
    table[0, 0] = n_pages
    first, end = rng.integers(-2, width, n_req), rng.integers(-2, width + 5, n_req)
    n_free = 4
    free = np.full(n_pages, -9, np.int32)
    want, wt = free[:n_free].tolist(), table.copy()
    for r in range(n_req):
        for p in range(max(first[r], 0), min(end[r], width)):
            if 0 <= table[r, p] < n_pages:
                want.append(int(table[r, p]))
                wt[r, p] = -1
    dt, df, nf = i32(table), i32(free), i32([n_free])
    jx.kv_release(i32(first), i32(end), dt, df, nf)
    assert int(nf) == len(want) and df[:len(want)].tolist() == want and np.array_equal(dt.cpu().numpy(), wt)
    assert (df[len(want):] == -9).all()


# ---- together ----------------------------------------------------------------------------------------------------------

def test_steps_of_a_served_request_in_a_graph():
    """Plan, norm and rotation, attention over the cache, search results joined, captured once and replayed with new inputs:
    every replay equals the eager calls."""
    heads, kv, dim, page, n_req = 8, 2, 64, 16, 5
    lens, new = i32([30, 1, 7, 100, 47]), i32([1, 1, 1, 1, 1])
    qkv = normal((n_req, heads + 2 * kv, dim), BF, 0)
    q, k, v = qkv.split([heads, kv, kv], 1)
    pages = 64
    cache = normal((2, pages, page, kv, dim), BF, 1)
    first = cache.clone()
    perm = torch.randperm(pages, generator=torch.Generator().manual_seed(2)).int().cuda()
    table = torch.full((n_req, 10), -1, dtype=torch.int32, device="cuda")
    for r, n in enumerate([2, 1, 1, 7, 3]):
        table[r, :n] = perm[r * 10:r * 10 + n]
    first_table = table.clone()
    free = perm[50:].contiguous()
    free = torch.cat([free, torch.full((50,), -1, dtype=torch.int32, device="cuda")])
    n_free = i32([14])
    angle = torch.rand((200, 32), generator=torch.Generator().manual_seed(3)) * 6
    cos, sin = angle.cos().cuda(), angle.sin().cuda()
    w = normal((dim,), BF, 4)
    keys, values = normal((40, kv, dim), BF, 5), normal((40, kv, dim), BF, 6)
    ids = torch.randint(-1, 40, (n_req, heads, 10), generator=torch.Generator().manual_seed(7), dtype=torch.int32).cuda()

    def step():
        plan = jx.kv_plan(lens, new, table, free, n_free, page, n_req)
        ready = jx.qk_norm_rope(q, k, v, cache[0], cache[1], plan.pos, plan.slot, cos, sin, w, w)
        part = jx.paged_attention(ready, cache[0], cache[1], table, plan.q_start, plan.kv_len, 0.125)
        out, lse = jx.found_attention(ready, keys, values, ids, 0.125, part=part)
        return out, lse, plan.kv_len

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(3):
        qkv.copy_(normal(qkv.shape, BF, 20 + i))
        lens.copy_(i32([30 + i, 1, 7, 96 + i, 47]))
        cache.copy_(first)
        table.copy_(first_table)  # no page belongs to two requests
        want = [x.clone() for x in step()]
        torch.cuda.synchronize()
        cache.copy_(first)
        table.copy_(first_table)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a, b)
