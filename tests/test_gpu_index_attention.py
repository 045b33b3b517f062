"""The example that decodes with a long past in an index: its steps before the past moves, and after, are attention over what the
cache and the search's result hold, from the definitions in 64 bits; pages go back and are used again."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

import attention_plain as plain  # noqa: E402
import index_attention as example  # noqa: E402


def check(server, got, k, v):
    """The last row against the keys [n][kv_heads][dim] of each head."""
    out, lse, ready, _ = got
    group = example.HEADS // example.KV_HEADS
    for h in range(example.HEADS):
        o, l, bo, bl = plain.attend_row(ready[-1, h].cpu().double(), k(h // group, h), v(h // group, h), server.scale, server.dtype)
        # where a part is joined with another it has been rounded to the element type on the way
        bo = bo + 2 * plain.UNIT[server.dtype] * v(h // group, h).abs().max()
        assert bool(((out[-1, h].cpu().double() - o).abs() <= bo).all()) and abs(float(lse[-1, h]) - l) <= 4 * bl


def test_steps_before_and_after_the_past_moves():
    past = 64 * example.PAGE
    server = example.Server(past, 100)
    for tokens in (500, past - 500 + 37):
        got = server.step(tokens)
    k, v = server.rows(0, past + 37)
    k, v = k.cpu().double(), v.cpu().double()
    check(server, got, lambda c, h: k[:, c], lambda c, h: v[:, c])
    free = int(server.n_free)
    server.move(past)
    assert int(server.n_free) == free + 64 and (server.table[0, :64] == -1).all()
    for step in range(20):
        got = server.step(1, k=16, L=64)
    n = past + 37 + 20
    assert int(server.len) == n
    rk, rv = server.rows(past, n)
    ids = got[3][0].cpu().long()
    pk, pv, rk, rv = (x.cpu().double() for x in (server.keys, server.values, rk, rv))
    assert (ids >= 0).all() and (ids < past).all()
    check(server, got, lambda c, h: torch.cat([rk[:, c], pk[ids[h], c]]), lambda c, h: torch.cat([rv[:, c], pv[ids[h], c]]))


def test_the_example_runs():
    worst, held = example.main(past=4000, steps=4, quiet=True)
    assert held > 0.5 and worst < 1.0
