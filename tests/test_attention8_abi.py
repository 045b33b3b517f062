"""The attention entry points over 8 bits without a GPU: records as the C compiler lays them out, refusals, and what the binding asks of
its tensors.  No kernel is launched."""
import ctypes as C
import os
import shutil
import subprocess

import pytest
import torch

from test_attention_abi import BAD_HEADS, HEX, ROOT, cache, jx, refused  # noqa: F401  (jx is the fixture)
from test_attention_limits import attend, found, rope  # noqa: F401
from test_attention_tensors import BF, F32, I32, I64, Stand, noted  # noqa: F401  (noted is a fixture)

E4, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def scales(jx, **kw):  # noqa: F811
    base = dict(d_k=HEX, d_v=HEX, block=16)
    base.update(kw)
    return C.byref(jx.KvScales(**base))


def calls(jx):  # noqa: F811
    return {
        "rope": lambda a, s: jx._lib.jx_qk_norm_rope8(C.byref(a), s, None),
        "attend": lambda a, s: jx._lib.jx_paged_attention8(C.byref(a), s, HEX, 1 << 40, None),
        "bytes": lambda a, s: jx._lib.jx_paged_attention8_bytes(C.byref(a), s),
        "found": lambda a, s: jx._lib.jx_found_attention8(C.byref(a), s, None),
    }


MAKE = {"rope": rope, "attend": attend, "bytes": attend, "found": found}


def test_record_matches_the_header(jx, tmp_path):  # noqa: F811
    cc = shutil.which("gcc") or shutil.which("cc")
    if not cc:
        pytest.skip("no C compiler")
    src = tmp_path / "sizes.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "jx.h"\nint main(void) {\n'
                   'printf("%zu %zu %zu %zu\\n", sizeof(jx_kv_scales), offsetof(jx_kv_scales, d_k), offsetof(jx_kv_scales, d_v), offsetof(jx_kv_scales, block));\n'
                   'return 0; }\n')
    exe = str(tmp_path / "sizes")
    subprocess.run([cc, "-I", os.path.join(ROOT, "include"), str(src), "-o", exe], check=True)
    got = [int(x) for x in subprocess.run([exe], check=True, capture_output=True, text=True).stdout.split()]
    s = jx.KvScales
    assert got == [C.sizeof(s), s.d_k.offset, s.d_v.offset, s.block.offset]


@pytest.mark.parametrize("call", ["rope", "attend", "bytes", "found"])
def test_refusals_of_all(jx, call):  # noqa: F811
    run, make = calls(jx)[call], MAKE[call]
    for bad in BAD_HEADS + [dict(head_dim=8), dict(head_dim=24), dict(head_dim=72), dict(head_dim=200)]:
        refused(jx, run(make(jx, **bad), scales(jx)))
    for bad in [dict(block=0), dict(block=-16), dict(block=3), dict(block=24), dict(block=128)]:
        refused(jx, run(make(jx), scales(jx, **bad)))
    refused(jx, run(make(jx), None))
    if call != "bytes":
        refused(jx, run(make(jx), scales(jx, d_k=None)))
        refused(jx, run(make(jx), scales(jx, d_v=None)))
        assert run(make(jx, n_tokens=0), scales(jx)) == 0
    else:
        assert run(make(jx), scales(jx)) >= 0


@pytest.mark.parametrize("call", ["rope", "attend", "bytes"])
def test_refusals_of_caches(jx, call):  # noqa: F811
    """Rows of codes lie on 16-byte boundaries: strides are multiples of 16 codes.  A block is no longer than a page."""
    run, make = calls(jx)[call], MAKE[call]
    for bad in [dict(page=0), dict(page=12), dict(page=8192), dict(n_pages=0), dict(d_k=None), dict(d_v=None), dict(d_k=HEX + 2), dict(d_v=HEX + 8),
                dict(page_stride=1032), dict(token_stride=72), dict(head_stride=8), dict(page_stride=-16), dict(token_stride=1 << 34)]:
        refused(jx, run(make(jx, cache=cache(jx, **bad)), scales(jx)))
    refused(jx, run(make(jx, cache=cache(jx, page=8)), scales(jx)))
    assert b"block" in jx._lib.jx_last_error()


def test_refusals_of_each(jx):  # noqa: F811
    run = calls(jx)
    for bad in [dict(rot_dim=-16), dict(rot_dim=8), dict(rot_dim=80), dict(n_pos=-1), dict(n_pos=1 << 40), dict(eps=-1.0), dict(eps=float("nan")),
                dict(d_q=None), dict(d_k=None), dict(d_v=None), dict(d_q_out=None), dict(d_pos=None), dict(d_slot=None), dict(d_cos=None),
                dict(d_sin=HEX + 4), dict(d_q_weight=HEX + 2), dict(k_token_stride=1), dict(v_head_stride=9), dict(q_head_stride=7)]:
        refused(jx, run["rope"](rope(jx, **bad), scales(jx)))
    for heads, kv, dim, tokens in ((1, 1, 256, 1 << 27), (32, 32, 256, 1 << 24), (8, 8, 64, 1 << 26), (1024, 1024, 16, 1 << 19)):
        refused(jx, run["rope"](rope(jx, n_heads=heads, n_kv_heads=kv, head_dim=dim, rot_dim=0, n_tokens=tokens), scales(jx)))
        assert b"n_tokens" in jx._lib.jx_last_error()
    for bad in [dict(d_q=None), dict(d_q=HEX + 4), dict(q_token_stride=12), dict(d_out=None), dict(d_q_start=None), dict(d_kv_len=None), dict(window=-1),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(table_pages=0), dict(table_pages=1 << 28), dict(n_req=-1), dict(n_req=1 << 28),
                dict(d_table=None)]:
        refused(jx, run["attend"](attend(jx, **bad), scales(jx)))
    need = jx._lib.jx_paged_attention8_bytes(C.byref(attend(jx)), scales(jx))
    if need:
        refused(jx, jx._lib.jx_paged_attention8(C.byref(attend(jx)), scales(jx), None, 0, None))
        refused(jx, jx._lib.jx_paged_attention8(C.byref(attend(jx)), scales(jx), HEX + 16, need, None))
        refused(jx, jx._lib.jx_paged_attention8(C.byref(attend(jx)), scales(jx), HEX, need - 1, None), -2)
    for bad in [dict(k=-1), dict(n_rows=-1), dict(n_rows=1 << 33), dict(d_part_out=HEX), dict(d_part_lse=HEX), dict(d_q=None), dict(d_out=None),
                dict(d_ids=None), dict(d_keys=None), dict(d_values=None), dict(d_keys=HEX + 8), dict(row_stride=136), dict(row_stride=-128),
                dict(head_stride=8), dict(d_part_out=HEX + 2, d_part_lse=HEX), dict(scale=float("nan")), dict(n_tokens=1 << 24, n_heads=32, n_kv_heads=1)]:
        refused(jx, run["found"](found(jx, **bad), scales(jx)))
    for fn in (jx._lib.jx_qk_norm_rope8, jx._lib.jx_found_attention8):
        refused(jx, fn(None, scales(jx), None))
    refused(jx, jx._lib.jx_paged_attention8(None, scales(jx), None, 0, None))
    refused(jx, jx._lib.jx_paged_attention8_bytes(None, scales(jx)))


def tensors():
    """name -> (function of the tensors, tensors by name)."""
    s = Stand
    paged = dict(k_cache=s(E4, 9, 16, 2, 64), v_cache=s(E4, 9, 16, 2, 64), k_scale=s(E8, 9, 2, 2), v_scale=s(E8, 9, 2, 2))
    return {
        "qk_norm_rope8": (lambda jx, t: jx.qk_norm_rope8(t["q"], t["k"], t["v"], t["k_cache"], t["v_cache"], t["k_scale"], t["v_scale"], t["pos"],
                                                         t["slot"], t["cos"], t["sin"], t["q_weight"], t["k_weight"], out=t["out"]),
                          dict(q=s(BF, 5, 4, 64), k=s(BF, 5, 2, 64), v=s(BF, 5, 2, 64), pos=s(I32, 5), slot=s(I64, 5), cos=s(F32, 99, 32),
                               sin=s(F32, 99, 32), q_weight=s(BF, 64), k_weight=s(BF, 64), out=s(BF, 5, 4, 64), **paged)),
        "paged_attention8": (lambda jx, t: jx.paged_attention8(t["q"], t["k_cache"], t["v_cache"], t["k_scale"], t["v_scale"], t["table"], t["q_start"],
                                                               t["kv_len"], 0.1, out=(t["out"], t["lse"]), work=t["work"]),
                             dict(q=s(BF, 5, 4, 64), table=s(I32, 3, 4), q_start=s(I32, 4), kv_len=s(I32, 3), out=s(BF, 5, 4, 64), lse=s(F32, 5, 4),
                                  work=s(torch.uint8, 1 << 20), **paged)),
        "found_attention8": (lambda jx, t: jx.found_attention8(t["q"], t["keys"], t["values"], t["k_scale"], t["v_scale"], t["ids"], 0.1, 8,
                                                               part=(t["part"], t["part_lse"]), out=(t["out"], t["lse"])),
                             dict(q=s(BF, 5, 4, 64), keys=s(E4, 20, 2, 64), values=s(E4, 20, 2, 64), k_scale=s(E8, 3, 2), v_scale=s(E8, 3, 2),
                                  ids=s(I32, 5, 4, 7), part=s(BF, 5, 4, 64), part_lse=s(F32, 5, 4), out=s(BF, 5, 4, 64), lse=s(F32, 5, 4))),
    }


@pytest.mark.parametrize("call", list(tensors()))
def test_tensors_of_one_device(noted, call):  # noqa: F811
    jx, lib = noted  # noqa: F811
    run, t = tensors()[call]
    run(jx, t)
    assert lib.made == ["jx_" + call]
    for x in t.values():
        x.at, x.device = 1, torch.device("cuda", 1)
    run(jx, t)
    assert lib.made == ["jx_" + call] * 2


@pytest.mark.parametrize("call,name", [(c, n) for c, (_, t) in tensors().items() for n in t])
@pytest.mark.parametrize("fault", ["elsewhere", "on the CPU", "of another type", "needs a gradient"])
def test_a_tensor_that_does_not_fit(noted, call, name, fault):  # noqa: F811
    jx, lib = noted  # noqa: F811
    run, tensors_of = tensors()[call]
    t = tensors_of[name]
    if fault == "needs a gradient":
        if t.dtype not in (BF, F32, E4, E8) or name in ("out", "lse"):
            pytest.skip("nothing that is learnt")
        t.requires_grad = True
    elif fault == "of another type":
        if name == "q":
            t.dtype = torch.float32
        else:
            t.dtype = torch.uint8 if t.dtype is not torch.uint8 else I32
    else:
        t.at = 1 if fault == "elsewhere" else -1
        t.device = torch.device("cuda", 1)
    with pytest.raises((AssertionError, KeyError)):
        run(jx, tensors_of)
    assert not lib.made


def test_scales_that_do_not_belong_to_the_cache(noted):  # noqa: F811
    jx, lib = noted  # noqa: F811
    for shape in ((9, 3, 2), (9, 0, 2), (8, 2, 2), (9, 2, 1), (9, 32, 2)):
        for name in ("qk_norm_rope8", "paged_attention8"):
            run, t = tensors()[name]
            t["k_scale"] = t["v_scale"] = Stand(E8, *shape)
            with pytest.raises(AssertionError):
                run(jx, t)
    run, t = tensors()["paged_attention8"]
    t["v_scale"] = Stand(E8, 9, 1, 2)
    with pytest.raises(AssertionError):
        run(jx, t)
    run, t = tensors()["found_attention8"]
    t["k_scale"] = Stand(E8, 2, 2)
    with pytest.raises(AssertionError):
        run(jx, t)
    assert not lib.made


def test_records_are_packed_as_they_are_declared(jx):  # noqa: F811
    def fields(cls, at=0):
        for name, kind in cls._fields_:
            off = at + getattr(cls, name).offset
            if issubclass(kind, C.Structure):
                yield from fields(kind, off)
            else:
                yield kind, off

    for packed, cls in ((jx._ROPE, jx.RopeArgs), (jx._ATTEND, jx.AttendArgs), (jx._FOUND, jx.FoundArgs), (jx._SCALES, jx.KvScales)):
        want = list(fields(cls))
        record = packed.pack(*[float(n + 1) if kind is C.c_float else n + 1 for n, (kind, _) in enumerate(want)])
        assert [kind.from_buffer_copy(record, off).value for kind, off in want] == list(range(1, len(want) + 1)), cls
