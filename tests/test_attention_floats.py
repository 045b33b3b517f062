"""Scales and epsilons that float32 does not hold, through the binding, without a GPU: a record of C's has an infinity there, which the library
refuses as a scale and takes as an epsilon."""
import ctypes as C
import math

import pytest

import test_attention8_abi
import test_attention_tensors
from test_attention_tensors import jx, noted  # noqa: F401  (fixtures)


def tensors(call):
    both = {**test_attention_tensors.calls(), **test_attention8_abi.tensors()}
    return both[call][1]


def run(jx, call, x):  # noqa: F811
    t = tensors(call)
    scales = (t["k_scale"], t["v_scale"]) if call.endswith("8") else ()
    if call.startswith("qk_norm_rope"):
        return getattr(jx, call)(t["q"], t["k"], t["v"], t["k_cache"], t["v_cache"], *scales, t["pos"], t["slot"], eps=x, out=t["out"])
    if call.startswith("paged"):
        return getattr(jx, call)(t["q"], t["k_cache"], t["v_cache"], *scales, t["table"], t["q_start"], t["kv_len"], x, out=(t["out"], t["lse"]),
                                 work=t["work"])
    return getattr(jx, call)(t["q"], t["keys"], t["values"], *scales, t["ids"], x, *((8,) if scales else ()), out=(t["out"], t["lse"]))


RECORDS = {"qk_norm_rope": ("RopeArgs", "eps"), "paged_attention": ("AttendArgs", "scale"), "found_attention": ("FoundArgs", "scale")}
CALLS = [x + y for x in RECORDS for y in ("", "8")]
VALUES = [0.1, 0.0, -2.5, 1e-300, 3.4028234e38, -3.4028235e38, 3.40282356e38, 1e39, -1e300, math.inf, -math.inf, math.nan]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("x", VALUES)
def test_a_record_has_what_float32_makes_of_it(noted, monkeypatch, call, x):  # noqa: F811
    jx, lib = noted  # noqa: F811
    got = []
    monkeypatch.setattr(jx, "_lib", type("Library", (), {"__getattr__": lambda self, name: lambda *args: got.append(args) or 0})())
    run(jx, call, x)
    record, field = RECORDS[call.rstrip("8")]
    value = getattr(getattr(jx, record).from_buffer_copy(got[-1][0]), field)
    want = C.c_float(x).value
    assert value == want or (math.isnan(value) and math.isnan(want))


@pytest.mark.parametrize("call", [x for x in CALLS if "rope" not in x])
@pytest.mark.parametrize("x", [1e39, -1e300, math.inf, math.nan])
def test_the_library_refuses_such_a_scale(jx, noted, monkeypatch, call, x):  # noqa: F811
    lib = jx.load_library()
    monkeypatch.setattr(jx, "_lib", lib)  # refused before anything is launched
    with pytest.raises(RuntimeError, match="scale"):
        run(jx, call, x)
