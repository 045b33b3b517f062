"""The example that decodes with a long past in an index, with keys and values of 8 bits: its steps before the past moves, and after,
are attention over what the cache and the search's result then hold, from the definitions in 64 bits; what has moved is what was held."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

import attention_plain as plain  # noqa: E402
import index_attention as example  # noqa: E402
from test_gpu_index_attention import check  # noqa: E402


def test_steps_before_and_after_the_past_moves():
    past = 64 * example.PAGE
    server = example.Server(past, 100, bits=8)
    for tokens in (500, past - 500 + 37):
        got = server.step(tokens)
    k, v = (x.cpu().double() for x in server.rows(0, past + 37))
    check(server, got, lambda c, h: k[:, c], lambda c, h: v[:, c])
    free = int(server.n_free)
    server.move(past)
    assert int(server.n_free) == free + 64 and (server.table[0, :64] == -1).all()
    pk, pv = (x.cpu().double() for x in server.past())
    assert torch.equal(pk, k[:past]) and torch.equal(pv, v[:past])
    for _ in range(20):  # one at a time, into blocks that hold others
        got = server.step(1, k=16, L=64)
    n = past + 37 + 20
    assert int(server.len) == n
    rk, rv = (x.cpu().double() for x in server.rows(past, n))
    ids = got[3][0].cpu().long()
    assert (ids >= 0).all() and (ids < past).all()
    check(server, got, lambda c, h: torch.cat([rk[:, c], pk[ids[h], c]]), lambda c, h: torch.cat([rv[:, c], pv[ids[h], c]]))


def test_8_bits_hold_what_16_bits_hold():
    """The same tokens: keys and values agree to half a step of e4m3 each, 2^-4 of a number or 2^-10 scales, and what comes before
    the rounding is computed alike.  Tokens arrive in chunks of whole blocks, so that each value is rounded once."""
    servers = [example.Server(512, 100, bits=bits) for bits in (16, 8)]
    for server in servers:
        for tokens in (256, 256):
            server.step(tokens)
    a, b = (s.rows(0, 512) for s in servers)
    scales = (x.float().repeat_interleave(example.BLOCK, 0)[..., None] for x in servers[1].held(0, 512)[2:])
    for x, y, scale in zip(a, b, scales):
        x, y, scale = x.double(), y.double(), scale.double()
        # the bfloat16 value is itself within 2^-8 of what both are rounded from
        size = x.abs() * (1 + 2.0 ** -7)
        half = torch.exp2(torch.floor(torch.log2((size / scale).clamp(min=2.0 ** -6))) - 4) * scale
        assert bool(((x - y).abs() <= half + 2.0 ** -8 * size).all())


def test_the_example_runs():
    worst, held = example.main(past=4000, steps=4, quiet=True, bits=8)
    assert held > 0.5 and worst < 1.0
