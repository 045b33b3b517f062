"""Which height the tiles of a call over 8 bits have, without a GPU.  It shows in the workspace: tiles of 64 rows are shared out over four workgroups on
each CU, those of 128 over two, each with a record of its own; and a call over 16 bits, which has no tiles of 64 rows, asks for as
much as one over 8 bits that takes 128."""
import ctypes as C

import pytest

from test_attention8_abi import scales
from test_attention_abi import cache, jx  # noqa: F401  (the fixture)
from test_attention_limits import attend


def low_tiles(jx, n_req, tokens, heads=8, **kw):  # noqa: F811
    """Whether the call takes tiles of 64 rows, by its workspace."""
    a = attend(jx, n_heads=heads, n_kv_heads=kw.pop("kv", heads), n_tokens=tokens, n_req=n_req, cache=cache(jx, page=8, page_stride=8 * 64 * heads, n_pages=1 << 16),
               table_pages=1 << 10, q_token_stride=64 * heads, **kw)
    coded, plain = jx._lib.jx_paged_attention8_bytes(C.byref(a), scales(jx, block=8)), jx._lib.jx_paged_attention_bytes(C.byref(a))
    assert coded >= 0 and plain >= 0
    return coded != plain


def test_the_workspace_shows_it(jx):  # noqa: F811
    assert low_tiles(jx, 33, 33 * 40)
    assert not low_tiles(jx, 33, 33 * 40, kv=2) and not low_tiles(jx, 33, 33 * 40, head_dim=128) and not low_tiles(jx, 2, 2000)


@pytest.mark.parametrize("n_req,mean", [(n, m) for n in (40, 150, 300, 450, 460, 500, 600, 680) for m in (33, 40, 50, 60, 64)])
def test_tiles_of_64_rows_where_four_workgroups_have_room_on_a_cu(jx, n_req, mean):  # noqa: F811
    """Keys and values of 64 elements take 32 KiB of a workgroup's LDS, the first rows and lengths of all requests and the units of all slots the rest of
    its quarter.  With more than 1,024 slots each tile is a share, and nothing but the keys and values is held (and no workspace asked for)."""
    slots = n_req * mean // 64 + n_req
    shares = 8 * (n_req + 1) + 4 * (slots + 1) + 2 * slots
    if slots <= 1024:
        assert low_tiles(jx, n_req, n_req * mean) == (shares <= 8192), (slots, shares)


@pytest.mark.parametrize("n_req", [1, 12, 33, 100, 300])
def test_tiles_of_64_rows_where_requests_have_as_many_on_the_mean(jx, n_req):  # noqa: F811
    """Alike chunks of 65 to 128 tokens are two tiles of 64 rows, of which the second reads all keys again, or one of 128."""
    for tokens, want in ((33 * n_req, True), (64 * n_req, True), (64 * n_req + 1, False), (65 * n_req, False), (96 * n_req, False), (128 * n_req, False),
                         (192 * n_req, False), (300 * n_req, False)):
        assert low_tiles(jx, n_req, tokens) == want, tokens
