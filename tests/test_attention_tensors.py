"""What the attention calls of the binding ask of their tensors, without a GPU: stand-ins for tensors on a device, and a library that
notes its calls."""
import contextlib

import pytest
import torch

from test_attention_abi import jx  # noqa: F401  (the fixture)


class Stand:
    """Shape, strides and device of a tensor that is nowhere."""
    is_cuda = True

    def __init__(self, dtype, *shape, device=0, strides=None):
        t = torch.empty(shape, dtype=dtype, device="meta")
        self.t, self.dtype, self.shape, self.strides, self.at = t, dtype, t.shape, strides or t.stride(), device
        self.device, self.requires_grad = torch.device("cuda", device), False

    def get_device(self):
        return self.at

    def stride(self, i=None):
        return tuple(self.strides) if i is None else self.strides[i]

    def is_contiguous(self):
        return tuple(self.strides) == self.t.stride()

    def data_ptr(self):
        return 4096


BF, I32, I64, F32 = torch.bfloat16, torch.int32, torch.int64, torch.float32


def calls():
    """name -> (function of the tensors, tensors by name)."""
    s = Stand
    cache = dict(k_cache=s(BF, 9, 16, 2, 64), v_cache=s(BF, 9, 16, 2, 64))
    return {
        "kv_plan": (lambda jx, t: jx.kv_plan(t["lens"], t["new"], t["table"], t["free"], t["n_free"], 16, 5, out=jx.KvPlan(
            t["q_start"], t["kv_len"], t["pos"], t["slot"], t["left"])),
            dict(lens=s(I32, 3), new=s(I32, 3), table=s(I32, 3, 4), free=s(I32, 9), n_free=s(I32, 1), q_start=s(I32, 4), kv_len=s(I32, 3),
                 pos=s(I32, 5), slot=s(I64, 5), left=s(I32, 1))),
        "kv_release": (lambda jx, t: jx.kv_release(t["first"], t["end"], t["table"], t["free"], t["n_free"]),
                       dict(first=s(I32, 3), end=s(I32, 3), table=s(I32, 3, 4), free=s(I32, 9), n_free=s(I32, 1))),
        "qk_norm_rope": (lambda jx, t: jx.qk_norm_rope(t["q"], t["k"], t["v"], t["k_cache"], t["v_cache"], t["pos"], t["slot"], t["cos"], t["sin"],
                                                       t["q_weight"], t["k_weight"], out=t["out"]),
                         dict(q=s(BF, 5, 4, 64), k=s(BF, 5, 2, 64), v=s(BF, 5, 2, 64), pos=s(I32, 5), slot=s(I64, 5), cos=s(F32, 99, 32),
                              sin=s(F32, 99, 32), q_weight=s(BF, 64), k_weight=s(BF, 64), out=s(BF, 5, 4, 64), **cache)),
        "paged_attention": (lambda jx, t: jx.paged_attention(t["q"], t["k_cache"], t["v_cache"], t["table"], t["q_start"], t["kv_len"], 0.1,
                                                             out=(t["out"], t["lse"]), work=t["work"]),
                            dict(q=s(BF, 5, 4, 64), table=s(I32, 3, 4), q_start=s(I32, 4), kv_len=s(I32, 3), out=s(BF, 5, 4, 64), lse=s(F32, 5, 4),
                                 work=s(torch.uint8, 1 << 20), **cache)),
        "found_attention": (lambda jx, t: jx.found_attention(t["q"], t["keys"], t["values"], t["ids"], 0.1, part=(t["part"], t["part_lse"]),
                                                             out=(t["out"], t["lse"])),
                            dict(q=s(BF, 5, 4, 64), keys=s(BF, 20, 2, 64), values=s(BF, 20, 2, 64), ids=s(I32, 5, 4, 7), part=s(BF, 5, 4, 64),
                                 part_lse=s(F32, 5, 4), out=s(BF, 5, 4, 64), lse=s(F32, 5, 4))),
    }


NAMES = [(call, name) for call, (_, tensors) in calls().items() for name in tensors]


@pytest.fixture
def noted(jx, monkeypatch):  # noqa: F811
    """The binding with a library that notes its calls."""
    class Library:
        made = []

        def __getattr__(self, name):
            return lambda *args: self.made.append(name) or 0

    lib = Library()
    lib.made.clear()
    monkeypatch.setattr(jx, "_lib", lib)
    monkeypatch.setattr(jx, "_raw_stream", lambda i: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "device", lambda i: contextlib.nullcontext())
    return jx, lib


@pytest.mark.parametrize("call", list(calls()))
def test_tensors_of_one_device(noted, call):
    jx, lib = noted
    run, tensors = calls()[call]
    run(jx, tensors)
    assert lib.made == ["jx_" + call]
    for t in tensors.values():
        t.at, t.device = 1, torch.device("cuda", 1)
    run(jx, tensors)
    assert lib.made == ["jx_" + call] * 2


@pytest.mark.parametrize("call,name", NAMES)
@pytest.mark.parametrize("device", [1, -1])
def test_a_tensor_that_is_elsewhere(noted, call, name, device):
    """On another GPU, or on none."""
    jx, lib = noted
    run, tensors = calls()[call]
    tensors[name].at, tensors[name].is_cuda, tensors[name].device = device, device >= 0, torch.device("cuda", 1) if device > 0 else torch.device("cpu")
    with pytest.raises(AssertionError):
        run(jx, tensors)
    assert not lib.made


LEARNT = [(call, name) for call, name in NAMES if name in
          ("q", "k", "v", "k_cache", "v_cache", "keys", "values", "q_weight", "k_weight", "cos", "sin", "part", "part_lse")]


@pytest.mark.parametrize("call,name", LEARNT)
def test_a_gradient_that_would_be_lost(noted, call, name):
    jx, lib = noted
    run, tensors = calls()[call]
    tensors[name].requires_grad = True
    with pytest.raises(AssertionError, match="gradient"):
        run(jx, tensors)
    assert not lib.made
    for mode in (torch.no_grad, torch.inference_mode):
        with mode():
            run(jx, tensors)
    assert lib.made == ["jx_" + call] * 2
