"""Sizes and arguments that the attention entry points refuse, without a GPU: no kernel is launched."""
import ctypes as C

import pytest

from test_attention_abi import HEX, cache, jx, refused  # noqa: F401  (jx is the fixture)


def attend(jx, **kw):
    base = dict(dtype=jx.BF16, n_heads=4, n_kv_heads=2, head_dim=64, n_tokens=3, d_q=HEX, q_token_stride=256, q_head_stride=64,
                cache=cache(jx), d_table=HEX, table_pages=8, n_req=2, d_q_start=HEX, d_kv_len=HEX, scale=0.1, window=0, d_out=HEX, d_lse=None)
    base.update(kw)
    return jx.AttendArgs(**base)


@pytest.mark.parametrize("page,table_pages", [(1, 0x7FFFFFFF), (16, (1 << 27) - 1), (4096, (1 << 19) - 1), (1, 0x7FFFFC01)])
def test_tables_that_end_beside_2_to_31(jx, page, table_pages):
    """The kernels look a few tiles ahead of the last key, in 32 bits."""
    c = cache(jx, page=page)
    if page * table_pages > 0x7FFFFC00:
        refused(jx, jx._lib.jx_paged_attention_bytes(C.byref(attend(jx, cache=c, table_pages=table_pages))))
        refused(jx, jx._lib.jx_paged_attention(C.byref(attend(jx, cache=c, table_pages=table_pages)), None, C.c_int64(0), None))
        refused(jx, jx._lib.jx_kv_plan(HEX, HEX, 2, page, HEX, table_pages, HEX, HEX, 9, 2 * HEX, HEX, 3 * HEX, HEX, HEX, 5, None))
        if page == 1:
            refused(jx, jx._lib.jx_kv_release(HEX, HEX, 1, HEX, table_pages, HEX, HEX, 9, None))
    largest = 0x7FFFFC00 // page
    assert jx._lib.jx_paged_attention_bytes(C.byref(attend(jx, cache=c, table_pages=largest))) >= 0


def found(jx, **kw):
    base = dict(dtype=jx.F16, n_heads=4, n_kv_heads=2, head_dim=64, n_tokens=3, d_q=HEX, q_token_stride=256, q_head_stride=64, d_keys=HEX,
                d_values=HEX, row_stride=128, head_stride=64, n_rows=5, d_ids=HEX, k=4, scale=0.1, d_part_out=None, d_part_lse=None, d_out=HEX,
                d_lse=None)
    base.update(kw)
    return jx.FoundArgs(**base)


@pytest.mark.parametrize("stride", [-128, -8, -(1 << 40)])
def test_found_rows_that_lie_backwards(jx, stride):
    """A negative offset stands for a row that is passed over."""
    refused(jx, jx._lib.jx_found_attention(C.byref(found(jx, row_stride=stride)), None))


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), -float("inf")])
def test_scales_that_are_not_finite(jx, scale):
    refused(jx, jx._lib.jx_paged_attention_bytes(C.byref(attend(jx, scale=scale))))
    refused(jx, jx._lib.jx_paged_attention(C.byref(attend(jx, scale=scale)), None, C.c_int64(0), None))
    refused(jx, jx._lib.jx_found_attention(C.byref(found(jx, scale=scale)), None))


@pytest.mark.parametrize("same", [dict(d_kv_len=HEX), dict(d_kv_len=5 * HEX)])
def test_plans_that_would_write_what_they_read(jx, same):
    """Every workgroup reads the lengths and the new tokens, and the first one writes the new lengths."""
    a = dict(d_len=HEX, d_new=5 * HEX, d_kv_len=3 * HEX)
    a.update(same)
    refused(jx, jx._lib.jx_kv_plan(a["d_len"], a["d_new"], 2, 16, HEX, 4, HEX, HEX, 9, 2 * HEX, HEX, a["d_kv_len"], HEX, HEX, 5, None))
    assert b"d_kv_len" in jx._lib.jx_last_error()


def rope(jx, **kw):
    base = dict(dtype=jx.BF16, n_heads=4, n_kv_heads=2, head_dim=64, rot_dim=32, interleaved=0, n_tokens=3, n_pos=10, d_q=HEX, d_k=HEX, d_v=HEX,
                q_token_stride=512, q_head_stride=64, k_token_stride=512, k_head_stride=64, v_token_stride=512, v_head_stride=64, d_q_weight=HEX,
                d_k_weight=None, eps=1e-6, d_cos=HEX, d_sin=HEX, d_pos=HEX, d_slot=HEX, d_q_out=HEX, cache=cache(jx))
    base.update(kw)
    return jx.RopeArgs(**base)


def test_calls_of_more_threads_than_a_launch_has(jx):
    """A launch has less than 2^32 threads: 64 for a list of found rows, 8 to 32 for a head (or four) of a token, 256 for a tile."""
    for heads, tokens in ((32, 1 << 21), (1, (1 << 26) - 3), (4096, 1 << 14)):
        refused(jx, jx._lib.jx_found_attention(C.byref(found(jx, n_heads=heads, n_kv_heads=1, n_tokens=tokens)), None))
        assert b"n_tokens" in jx._lib.jx_last_error()
    for heads, kv, dim, tokens in ((1, 1, 256, 1 << 27), (32, 32, 256, 1 << 24), (8, 8, 64, 1 << 27 >> 1), (64, 64, 128, (1 << 32) // (48 * 16) + 1)):
        refused(jx, jx._lib.jx_qk_norm_rope(C.byref(rope(jx, n_heads=heads, n_kv_heads=kv, head_dim=dim, n_tokens=tokens)), None))
        assert b"n_tokens" in jx._lib.jx_last_error()
    for n_req, kv in ((1 << 23, 2), ((1 << 23) + 1, 1), (1 << 20, 16)):
        a = attend(jx, n_req=n_req, n_heads=16, n_kv_heads=kv)
        refused(jx, jx._lib.jx_paged_attention_bytes(C.byref(a)))
        refused(jx, jx._lib.jx_paged_attention(C.byref(a), None, C.c_int64(0), None))
        assert b"n_req" in jx._lib.jx_last_error()
    assert jx._lib.jx_paged_attention_bytes(C.byref(attend(jx, n_req=1 << 22, n_kv_heads=2))) >= 0
