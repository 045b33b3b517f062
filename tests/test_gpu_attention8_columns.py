"""Attention of few rows over keys and values of 8 bits where the wavefronts of a workgroup share neighbouring key heads between them: two or four of
them, which it takes from as many units of 32 keys on as the launch has wavefronts.  Against the definition in 64 bits, bounds as in
attention_plain, for every key head."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2601_07048_amd import jx  # noqa: E402

import attention_plain as plain  # noqa: E402
from test_gpu_attention import BF, TYPES, i32  # noqa: E402
from test_gpu_attention8 import NAN_CODE, NAN_SCALE, Paged8  # noqa: E402


def wavefronts(dim):
    """Of a launch."""
    return 4096 if dim <= 64 else 2048 if dim <= 128 else 1024


def columns(kv):
    return 4 if kv % 4 == 0 else 2 if kv % 2 == 0 else 1


def units(p, window=0):
    """Of all key heads, at least: every request has as many units of 32 keys as its rows see."""
    new = torch.diff(p.q_start).tolist()
    room = p.table.shape[1] * p.page
    return p.k.shape[2] * sum(max(min(n, window + m if window else n, room) // 32, 1) for n, m in zip(p.kv_len.tolist(), new) if m)


def some_rows(p, rng, most):
    """The first and the last row, those of the longest and of the shortest request, and others."""
    start = p.q_start.tolist()
    at = sorted((n, r) for r, n in enumerate(p.kv_len.tolist()) if start[r + 1] > start[r])
    rows = {0, p.q.shape[0] - 1, start[at[0][1]], start[at[-1][1]], start[at[-1][1] + 1] - 1}
    return sorted(rows | set(rng.integers(0, p.q.shape[0], most - len(rows)).tolist()))


# query heads of a key head, key heads, dimension, page, block
CASES = [(2, 16, 64, 16, 16), (1, 8, 64, 32, 8), (4, 4, 64, 16, 1), (3, 8, 48, 64, 64), (4, 8, 128, 16, 16), (1, 16, 128, 128, 32), (5, 4, 96, 16, 4), (7, 4, 80, 32, 32),
         (4, 8, 256, 16, 16), (2, 16, 192, 64, 2), (3, 4, 208, 16, 16), (8, 2, 64, 16, 8), (2, 6, 128, 32, 16), (4, 2, 256, 16, 16)]


def lengths(kv, dim, times, rng, n_req=23):
    """Requests of unlike lengths, some of next to nothing, of at least `times` as many units as there are wavefronts."""
    short = [0, 1, 31, 32, 33, 64, 95]
    keys = int(times * 32 * wavefronts(dim)) // kv + 32 * n_req
    lens = short + [int(x) + 1 for x in rng.dirichlet(np.full(n_req - len(short), 0.7)) * keys]
    return [lens[i] for i in rng.permutation(n_req)]


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("group,kv,dim,page,block", CASES)
@pytest.mark.parametrize("times", [1, 2.7])
def test_key_heads_that_share_a_workgroup(dtype, group, kv, dim, page, block, times):
    rng = np.random.default_rng(dim + kv)
    lens = lengths(kv, dim, times, rng)
    p = Paged8(dtype, group * kv, kv, dim, page, block, lens, [1] * len(lens), seed=dim + kv, pad=2)
    assert columns(kv) > 1 and units(p) >= wavefronts(dim)
    p.check(rows=some_rows(p, rng, 9))
    p.check(window=100, rows=some_rows(p, rng, 9))  # fewer units than wavefronts, most of them


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("kv,dim,window", [(8, 64, 1100), (4, 128, 2000), (16, 96, 400), (8, 256, 150), (2, 128, 4000)])
def test_windows(dtype, kv, dim, window):
    rng = np.random.default_rng(window)
    n_req = max(32 * wavefronts(dim) // (kv * window) + 3, 320 // kv if window < 2000 else 0)  # too many tiles for a workgroup each
    lens = [int(x) for x in rng.integers(window + 64, window + 600, n_req)]
    p = Paged8(dtype, 2 * kv, kv, dim, 16, 8, lens, [1] * n_req, seed=window)
    assert units(p, window) >= wavefronts(dim)
    p.check(window=window, rows=some_rows(p, rng, 7))


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("group,kv,dim", [(4, 8, 64), (3, 4, 128), (2, 4, 256), (4, 2, 128)])
@pytest.mark.parametrize("new", [2, 5, 12])
def test_a_few_tokens_each(dtype, group, kv, dim, new):
    """Tiles of 16 rows that follow one another; of 32 where the cache has little room for each request."""
    rng = np.random.default_rng(new + dim)
    n_req = 32 * wavefronts(dim) // (kv * 200) + 1
    lens = [int(x) for x in rng.integers(200, 320, n_req)]
    p = Paged8(dtype, group * kv, kv, dim, 16, 4, lens, [1 + r % new for r in range(n_req)], seed=new, width=64)
    assert units(p) >= wavefronts(dim)
    p.check(rows=some_rows(p, rng, 9))
    p.check(window=230, rows=some_rows(p, rng, 9))


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("kv,dim", [(16, 64), (4, 128), (8, 256), (2, 128)])
def test_tables_with_holes(dtype, kv, dim):
    rng = np.random.default_rng(kv)
    lens = lengths(kv, dim, 1.5, rng)
    p = Paged8(dtype, kv, kv, dim, 16, 16, lens, [1] * len(lens), seed=kv)
    n = int(np.argmax(lens))
    holes = torch.from_numpy(rng.random(p.table.shape) < 0.3).cuda()
    p.table[holes] = -1
    p.table[n, 1], p.table[n, 2], p.table[n, lens[n] // 32] = p.k.shape[0], 2 ** 31 - 1, -(2 ** 31)
    p.check(rows=some_rows(p, rng, 9))
    p.table[n] = -1  # the longest sees nothing
    got = p.check(rows=some_rows(p, rng, 9))
    assert (got[1][n] == -math.inf).all() and not got[0][n].any()
    p.table = p.table[:, :max(lens) // 48].contiguous()  # narrower than some lengths
    p.check(rows=some_rows(p, rng, 9))


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("kv,dim", [(8, 64), (4, 128), (16, 128), (8, 256), (2, 128)])
@pytest.mark.parametrize("what", ["code", "scale"])
def test_what_is_not_a_number_stays_in_its_head(dtype, kv, dim, what):
    """In the last key head, at the first key, one in the middle, the last: of those that see it this head's results alone are none; where the
    window has left it behind, everything is as it is without it."""
    rng = np.random.default_rng(kv + dim)
    group, block = 2, 8
    lens = lengths(kv, dim, 1.3, rng)
    p = Paged8(dtype, group * kv, kv, dim, 16, block, lens, [1] * len(lens), seed=kv)
    n = int(np.argmax(lens))
    rows = sorted({0, n, len(lens) - 1, int(np.argsort(lens)[-2])})
    want, want_window = p.want(rows=rows), p.want(window=500, rows=rows)
    for at in (0, lens[n] // 2, lens[n] - 501 - block, lens[n] - 501, lens[n] - 1):
        page, place = p.place(n, at)
        for codes, scale in ((p.v, p.v_scale), (p.k, p.k_scale)):
            bad = codes.view(torch.uint8)[page, place, kv - 1, 3:4] if what == "code" else scale.view(torch.uint8)[page, place // block, kv - 1:kv]
            keep = bad.clone()
            bad.fill_(NAN_CODE if what == "code" else NAN_SCALE)
            out, lse = p.run()
            hidden = torch.zeros_like(out, dtype=torch.bool)
            if codes is p.v and what == "code":
                hidden[n, -group:, 3] = True
            else:
                hidden[n, -group:] = True
            assert out[hidden].isnan().all() and torch.isfinite(out[~hidden]).all(), at
            if codes is p.k:
                assert lse[n, -group:].isnan().all()
            plain.check((out, lse), {x: y for x, y in want.items() if not hidden[x].any()}, at)
            got = p.run(window=500)
            if (at if what == "code" else at // block * block + block - 1) < lens[n] - 500:  # a scale is that of the whole block
                plain.check(got, want_window, (at, "window"))
            bad.copy_(keep)


@pytest.mark.parametrize("dtype", TYPES, ids=["bf16", "f16"])
@pytest.mark.parametrize("kv,dim", [(8, 64), (4, 128), (8, 256)])
def test_the_same_bits_whatever_the_workspace_held(dtype, kv, dim):
    rng = np.random.default_rng(kv + dim)
    lens = lengths(kv, dim, 2, rng)
    p = Paged8(dtype, 4 * kv, kv, dim, 16, 16, lens, [1] * len(lens), seed=kv)
    want = p.run()
    work = torch.zeros(1 << 28, dtype=torch.uint8, device="cuda")
    for fill in (0, 0xFF, 0x7F):
        work.fill_(fill)
        got = p.run(work=work, out=(torch.full_like(want[0], math.nan), torch.full_like(want[1], math.nan)))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), fill


def test_a_graph_whose_lengths_change_what_is_shared():
    """Captured where a column each has keys enough; replayed with lengths that have too few, and with the first ones."""
    kv, dim = 8, 128
    rng = np.random.default_rng(3)
    lens = lengths(kv, dim, 2, rng)
    p = Paged8(BF, 2 * kv, kv, dim, 16, 16, lens, [1] * len(lens), seed=1)
    p.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = jx.paged_attention8(p.q, p.k, p.v, p.k_scale, p.v_scale, p.table, p.q_start, p.kv_len, p.scale)
    for now in (lens, [min(n, 40) for n in lens], [n // 3 for n in lens], lens):
        p.kv_len.copy_(i32(now))
        want = p.run()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held[0], want[0]) and torch.equal(held[1], want[1])
        plain.check(held, p.want(rows=[0, 5, 11]))
