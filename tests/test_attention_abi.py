"""The attention entry points without a GPU: argument records as the C compiler lays them out, and refusals.  No kernel is launched."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def jx():
    if not os.path.exists(os.path.join(ROOT, "paper_2601_07048_amd", "libjx.so")):
        import __graft_entry__
        __graft_entry__.build()
    from paper_2601_07048_amd import jx
    return jx


def test_records_match_the_header(jx, tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if not cc:
        pytest.skip("no C compiler")
    pairs = [("jx_kv_cache", jx.KvCache), ("jx_rope_args", jx.RopeArgs), ("jx_attend_args", jx.AttendArgs), ("jx_found_args", jx.FoundArgs)]
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "jx.h"', "int main(void) {"]
    want = []
    for name, cls in pairs:
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        want.append(C.sizeof(cls))
        for field, _ in cls._fields_:
            lines.append(f'printf("%zu\\n", offsetof({name}, {field}));')
            want.append(getattr(cls, field).offset)
    src = tmp_path / "sizes.c"
    src.write_text("\n".join(lines + ["return 0; }"]))
    exe = str(tmp_path / "sizes")
    subprocess.run([cc, "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    got = [int(x) for x in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()]
    assert got == want


HEX = 4096  # an aligned address that nothing reads: every call here is refused before it launches


def refused(jx, rc, code=-1):
    assert rc == code, (rc, jx._lib.jx_last_error())
    assert jx._lib.jx_last_error()


def cache(jx, **kw):
    base = dict(d_k=HEX, d_v=HEX, page_stride=1024, token_stride=64, head_stride=64, page=16, n_pages=4)
    base.update(kw)
    return jx.KvCache(**base)


BAD_CACHES = [dict(page=0), dict(page=12), dict(page=8192), dict(n_pages=0), dict(d_k=None), dict(d_v=None), dict(d_k=HEX + 2), dict(d_v=HEX + 8),
              dict(page_stride=4), dict(token_stride=65), dict(head_stride=3)]
BAD_HEADS = [dict(dtype=1), dict(dtype=0), dict(dtype=9), dict(n_heads=0), dict(n_heads=3, n_kv_heads=2), dict(n_kv_heads=0), dict(n_heads=2, n_kv_heads=4),
             dict(head_dim=0), dict(head_dim=12), dict(head_dim=264), dict(n_tokens=-1), dict(n_tokens=1 << 40), dict(n_heads=8192, n_kv_heads=1)]


def test_attention_refusals(jx):
    def args(**kw):
        base = dict(dtype=jx.BF16, n_heads=4, n_kv_heads=2, head_dim=64, n_tokens=3, d_q=HEX, q_token_stride=256, q_head_stride=64,
                    cache=cache(jx), d_table=HEX, table_pages=8, n_req=2, d_q_start=HEX, d_kv_len=HEX, scale=0.1, window=0, d_out=HEX, d_lse=None)
        base.update(kw)
        return jx.AttendArgs(**base)

    call = lambda a: jx._lib.jx_paged_attention(C.byref(a), None, C.c_int64(0), None)  # noqa: E731
    sized = BAD_HEADS + [dict(cache=cache(jx, **c)) for c in BAD_CACHES] + \
        [dict(table_pages=0), dict(table_pages=1 << 28), dict(n_req=-1), dict(n_req=1 << 28), dict(d_table=None), dict(window=-1)]
    for bad in sized:
        refused(jx, call(args(**bad)))
        refused(jx, jx._lib.jx_paged_attention_bytes(C.byref(args(**bad))))
    for bad in [dict(d_q=None), dict(d_q=HEX + 4), dict(q_token_stride=12), dict(q_head_stride=2), dict(d_out=None), dict(d_out=HEX + 2),
                dict(d_q_start=None), dict(d_kv_len=None)]:
        refused(jx, call(args(**bad)))
    refused(jx, jx._lib.jx_paged_attention(None, None, C.c_int64(0), None))
    refused(jx, jx._lib.jx_paged_attention_bytes(None))
    assert jx._lib.jx_paged_attention_bytes(C.byref(args())) >= 0
    assert call(args(n_tokens=0)) == 0
    need = jx._lib.jx_paged_attention_bytes(C.byref(args()))
    if need:
        refused(jx, call(args()))
        refused(jx, jx._lib.jx_paged_attention(C.byref(args()), C.c_void_p(HEX + 16), C.c_int64(need), None))
        refused(jx, jx._lib.jx_paged_attention(C.byref(args()), C.c_void_p(HEX), C.c_int64(need - 1), None), -2)


def test_found_refusals(jx):
    def args(**kw):
        base = dict(dtype=jx.F16, n_heads=4, n_kv_heads=2, head_dim=64, n_tokens=3, d_q=HEX, q_token_stride=256, q_head_stride=64, d_keys=HEX,
                    d_values=HEX, row_stride=128, head_stride=64, n_rows=5, d_ids=HEX, k=4, scale=0.1, d_part_out=None, d_part_lse=None, d_out=HEX,
                    d_lse=None)
        base.update(kw)
        return jx.FoundArgs(**base)

    call = lambda a: jx._lib.jx_found_attention(C.byref(a), None)  # noqa: E731
    for bad in BAD_HEADS + [dict(k=-1), dict(n_rows=-1), dict(n_rows=1 << 33), dict(d_part_out=HEX), dict(d_part_lse=HEX), dict(d_q=None),
                            dict(q_head_stride=12), dict(d_out=None), dict(d_ids=None), dict(d_keys=None), dict(d_values=None), dict(d_keys=HEX + 8),
                            dict(row_stride=100), dict(head_stride=4), dict(d_part_out=HEX + 2, d_part_lse=HEX)]:
        refused(jx, call(args(**bad)))
    refused(jx, jx._lib.jx_found_attention(None, None))
    assert call(args(n_tokens=0)) == 0


def test_rope_refusals(jx):
    def args(**kw):
        base = dict(dtype=jx.BF16, n_heads=4, n_kv_heads=2, head_dim=64, rot_dim=32, interleaved=0, n_tokens=3, n_pos=10, d_q=HEX, d_k=HEX, d_v=HEX,
                    q_token_stride=512, q_head_stride=64, k_token_stride=512, k_head_stride=64, v_token_stride=512, v_head_stride=64, d_q_weight=HEX,
                    d_k_weight=None, eps=1e-6, d_cos=HEX, d_sin=HEX, d_pos=HEX, d_slot=HEX, d_q_out=HEX, cache=cache(jx))
        base.update(kw)
        return jx.RopeArgs(**base)

    call = lambda a: jx._lib.jx_qk_norm_rope(C.byref(a), None)  # noqa: E731
    for bad in BAD_HEADS + [dict(cache=cache(jx, **c)) for c in BAD_CACHES] + \
            [dict(rot_dim=-16), dict(rot_dim=8), dict(rot_dim=80), dict(n_pos=-1), dict(n_pos=1 << 40), dict(eps=-1.0), dict(eps=float("nan")),
             dict(d_q=None), dict(d_k=None), dict(d_v=None), dict(d_q_out=None), dict(d_pos=None), dict(d_slot=None), dict(d_cos=None),
             dict(d_sin=None), dict(d_sin=HEX + 4), dict(d_q_weight=HEX + 2), dict(d_k_weight=HEX + 8), dict(k_token_stride=1),
             dict(v_head_stride=9), dict(q_head_stride=7)]:
        refused(jx, call(args(**bad)))
    refused(jx, jx._lib.jx_qk_norm_rope(None, None))
    assert call(args(n_tokens=0)) == 0


def test_plan_refusals(jx):
    names = ["d_len", "d_new", "n_req", "page", "d_table", "table_pages", "d_free", "d_n_free", "n_pages", "d_n_free_out", "d_q_start", "d_kv_len",
             "d_pos", "d_slot", "n_tokens"]
    ints = {"n_req": C.c_int32, "page": C.c_int32, "table_pages": C.c_int32, "n_pages": C.c_int32, "n_tokens": C.c_int64}

    def call(**kw):
        base = {n: HEX for n in names}
        base.update(n_req=2, page=16, table_pages=4, n_pages=9, n_tokens=5, d_n_free_out=2 * HEX)
        base.update(kw)
        return jx._lib.jx_kv_plan(*[ints.get(n, C.c_void_p)(base[n]) for n in names], None)

    for bad in [dict(page=0), dict(page=24), dict(n_pages=0), dict(table_pages=0), dict(table_pages=1 << 28), dict(n_req=-1), dict(n_req=8193),
                dict(n_tokens=-1), dict(n_tokens=1 << 31), dict(d_n_free_out=HEX)] + [{n: None} for n in names if n not in ints]:
        refused(jx, call(**bad))
    give = lambda *a: jx._lib.jx_kv_release(*a, None)  # noqa: E731
    p, i = C.c_void_p, C.c_int32
    refused(jx, give(p(HEX), p(HEX), i(1), p(HEX), i(4), p(HEX), p(HEX), i(0)))
    refused(jx, give(p(HEX), p(HEX), i(1), p(HEX), i(0), p(HEX), p(HEX), i(4)))
    refused(jx, give(p(HEX), p(HEX), i(8193), p(HEX), i(4), p(HEX), p(HEX), i(4)))
    refused(jx, give(p(HEX), p(HEX), i(-1), p(HEX), i(4), p(HEX), p(HEX), i(4)))
    for k in range(5):
        a = [p(HEX)] * 5
        a[k] = p(None)
        refused(jx, give(a[0], a[1], i(1), a[2], i(4), a[3], a[4], i(4)))
    assert give(p(HEX), p(HEX), i(0), p(HEX), i(4), p(HEX), p(HEX), i(4)) == 0
