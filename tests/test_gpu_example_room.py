"""The example keeps a request's past where a step finds no room."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

import index_attention as example  # noqa: E402
from test_gpu_index_attention import check  # noqa: E402


def test_a_step_without_room_forgets_nothing():
    server = example.Server(1024, 100)
    server.step(1024)
    pages = server.n_free
    server.n_free = torch.zeros_like(pages)
    out, lse, _, _ = server.step(1)  # the last page is full
    assert not out.any() and (lse == -float("inf")).all()
    assert int(server.len) == 1024 and int(server.n_free) == 0
    server.n_free = pages
    got = server.step(1)
    assert int(server.len) == 1025 and int(server.n_free) == int(pages) - 1
    k, v = (x.cpu().double() for x in server.rows(0, 1025))
    check(server, got, lambda c, h: k[:, c], lambda c, h: v[:, c])
