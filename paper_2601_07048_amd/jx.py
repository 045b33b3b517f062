"""Thin ctypes binding of libjx's C ABI (include/jx.h).

Argument marshalling only: every function here forwards torch tensors' device
pointers and the current HIP stream to the entry point of the same name.  There
is no CPU path; importing this module without a built ``libjx.so`` raises.

The library is loaded from this directory; the environment variable ``JX_LIB`` names another build of it (a development
aid for comparing builds; it changes which file is loaded, nothing else).
"""
from __future__ import annotations

import ctypes as C
import os
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("JX_LIB", os.path.join(_HERE, "libjx.so"))

NONE = 0xFFFFFFFF
U8, F32, F16, BF16 = 0, 1, 2, 3
EXACT, RABITQ = 0, 1
CAND_FRONTIER, CAND_VISITED = 0, 1
RULE_MAXCOS, RULE_MAXABS, RULE_DEFAULT = 0, 1, -1
# jx_params.flags / jx_set_flags (see include/jx.h)
FLAG_NO_PAIR, FLAG_NO_INCR_PRUNE, FLAG_NO_GRAM, FLAG_GRAM_U8 = 1 << 0, 1 << 1, 1 << 2, 1 << 3
FLAG_VISITED_IDS, FLAG_VISITED_NONE, FLAG_LANES_WIDE, FLAG_LANES_NARROW = 1 << 4, 1 << 5, 1 << 6, 1 << 7
FLAG_TILED_LOADS, FLAG_WAVES_2, FLAG_WAVES_4, FLAG_QPW_2, FLAG_QPW_4 = 1 << 8, 1 << 9, 1 << 10, 1 << 11, 1 << 12
MAX_L, MAX_R, MAX_BF_K = 512, 256, 128
MAX_REQUESTS, MAX_HEAD_DIM = 8192, 256

EXPORTS = [
    "jx_arena_bytes", "jx_create", "jx_destroy", "jx_insert", "jx_quantize", "jx_search", "jx_beam_frontier",
    "jx_bruteforce", "jx_size", "jx_export_graph", "jx_import_graph", "jx_export_codes", "jx_import_codes", "jx_rotate",
    "jx_rotate_points", "jx_encode_rotated", "jx_delete", "jx_consolidate", "jx_compact", "jx_deleted_count", "jx_probe_gather", "jx_mips_augment", "jx_strerror", "jx_last_error",
    "jx_bruteforce_static", "jx_bruteforce_kernel", "jx_set_flags",
    "jx_kv_plan", "jx_kv_release", "jx_qk_norm_rope", "jx_paged_attention_bytes", "jx_paged_attention", "jx_found_attention",
]


class Params(C.Structure):
    _fields_ = [
        ("dim", C.c_int32), ("dtype", C.c_int32), ("R", C.c_int32), ("L_build", C.c_int32), ("alpha", C.c_float),
        ("cand_mode", C.c_int32), ("capacity", C.c_int64), ("max_batch", C.c_int64), ("quant_bits", C.c_int32),
        ("batch_growth", C.c_float), ("flags", C.c_uint32),
    ]


class Stats(C.Structure):
    _fields_ = [("hops", C.c_uint64), ("dist_evals", C.c_uint64), ("adj_bytes", C.c_uint64),
                ("vec_bytes", C.c_uint64), ("rerank_bytes", C.c_uint64), ("rotate_ms", C.c_float),
                ("prep_ms", C.c_float), ("beam_ms", C.c_float), ("rerank_ms", C.c_float), ("beam_kernel", C.c_char * 96)]

    def as_dict(self):
        out = {k: (float if k.endswith("_ms") else int)(getattr(self, k)) for k, _ in self._fields_ if k != "beam_kernel"}
        out["beam_kernel"] = self.beam_kernel.decode()
        return out


class KvCache(C.Structure):
    _fields_ = [("d_k", C.c_void_p), ("d_v", C.c_void_p), ("page_stride", C.c_int64), ("token_stride", C.c_int64),
                ("head_stride", C.c_int64), ("page", C.c_int32), ("n_pages", C.c_int32)]


class RopeArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("n_tokens", C.c_int64), ("n_pos", C.c_int64),
                ("d_q", C.c_void_p), ("d_k", C.c_void_p), ("d_v", C.c_void_p),
                ("q_token_stride", C.c_int64), ("q_head_stride", C.c_int64), ("k_token_stride", C.c_int64),
                ("k_head_stride", C.c_int64), ("v_token_stride", C.c_int64), ("v_head_stride", C.c_int64),
                ("d_q_weight", C.c_void_p), ("d_k_weight", C.c_void_p), ("eps", C.c_float), ("d_cos", C.c_void_p),
                ("d_sin", C.c_void_p), ("d_pos", C.c_void_p), ("d_slot", C.c_void_p), ("d_q_out", C.c_void_p), ("cache", KvCache)]


class AttendArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("n_tokens", C.c_int64), ("d_q", C.c_void_p), ("q_token_stride", C.c_int64), ("q_head_stride", C.c_int64),
                ("cache", KvCache), ("d_table", C.c_void_p), ("table_pages", C.c_int32), ("n_req", C.c_int32),
                ("d_q_start", C.c_void_p), ("d_kv_len", C.c_void_p), ("scale", C.c_float), ("window", C.c_int32),
                ("d_out", C.c_void_p), ("d_lse", C.c_void_p)]


class FoundArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("n_tokens", C.c_int64), ("d_q", C.c_void_p), ("q_token_stride", C.c_int64), ("q_head_stride", C.c_int64),
                ("d_keys", C.c_void_p), ("d_values", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64),
                ("n_rows", C.c_int64), ("d_ids", C.c_void_p), ("k", C.c_int32), ("scale", C.c_float),
                ("d_part_out", C.c_void_p), ("d_part_lse", C.c_void_p), ("d_out", C.c_void_p), ("d_lse", C.c_void_p)]


class KvPlan(NamedTuple):
    """What jx_kv_plan writes beside the table."""
    q_start: torch.Tensor
    kv_len: torch.Tensor
    pos: torch.Tensor
    slot: torch.Tensor
    n_free: torch.Tensor


class JxError(RuntimeError):
    def __init__(self, code, text):
        super().__init__(f"libjx error {code}: {text}")
        self.code = code


def load_library(path: str = LIB_PATH) -> C.CDLL:
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python -m paper_2601_07048_amd.build` "
                          "(there is no CPU fallback)")
    lib = C.CDLL(path)
    lib.jx_arena_bytes.restype = C.c_int64
    lib.jx_strerror.restype = C.c_char_p
    lib.jx_last_error.restype = C.c_char_p
    lib.jx_bruteforce_kernel.restype = C.c_char_p
    lib.jx_paged_attention_bytes.restype = C.c_int64
    p, i, n = C.c_void_p, C.c_int32, C.c_int64
    lib.jx_kv_plan.argtypes = [p, p, i, i, p, i, p, p, i, p, p, p, p, p, n, p]
    lib.jx_kv_release.argtypes = [p, p, i, p, i, p, p, i, p]
    lib.jx_qk_norm_rope.argtypes = lib.jx_found_attention.argtypes = [p, p]
    lib.jx_paged_attention_bytes.argtypes = [p]
    lib.jx_paged_attention.argtypes = [p, p, n, p]
    for name in EXPORTS:
        getattr(lib, name)  # fail loudly on a missing symbol
    return lib


_lib = load_library()


def _check(rc):
    if rc != 0:
        raise JxError(rc, (_lib.jx_last_error() or b"").decode() or _lib.jx_strerror(rc).decode())


def _ptr(t):
    if t is None:
        return C.c_void_p(0)
    assert t.is_cuda and t.is_contiguous()
    return C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


# the stream's handle without an object around it (0.1 instead of 2.8 us)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)


def _torch_dtype(dtype):
    return {U8: torch.uint8, F32: torch.float32, F16: torch.float16}[dtype]


def jx_arena_bytes(params: Params) -> int:
    n = _lib.jx_arena_bytes(C.byref(params))
    if n < 0:
        _check(int(n))
    return int(n)


class Index:
    """Owns the arena tensor and the opaque handle; methods mirror the C ABI."""

    def __init__(self, dim, dtype, R, L_build, alpha=1.2, capacity=0, max_batch=0, quant_bits=0, batch_growth=0.25,
                 device="cuda:0", flags=0, cand_mode=CAND_FRONTIER, arena_bytes=0):
        self.params = Params(dim=dim, dtype=dtype, R=R, L_build=L_build, alpha=alpha, cand_mode=cand_mode,
                             capacity=capacity, max_batch=max_batch or capacity, quant_bits=quant_bits, batch_growth=batch_growth,
                             flags=flags)
        self.device = torch.device(device)
        self.dim, self.dtype, self.R = dim, dtype, R
        nbytes = arena_bytes or jx_arena_bytes(self.params)  # fewer: without byte copies (see jx_create)
        with torch.cuda.device(self.device):
            self.arena = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
            h = C.c_void_p()
            _check(_lib.jx_create(C.byref(self.params), _ptr(self.arena), C.c_int64(nbytes), _stream(), C.byref(h)))
        self._h = h

    def close(self):
        if getattr(self, "_h", None) and _lib is not None:  # _lib is gone at interpreter shutdown
            _lib.jx_destroy(self._h)
            self._h = None

    def __del__(self):
        self.close()

    # -- jx_set_flags
    def set_flags(self, flags):
        _check(_lib.jx_set_flags(self._h, C.c_uint32(flags)))

    # -- jx_size
    def size(self):
        n = C.c_int64()
        e = C.c_uint32()
        _check(_lib.jx_size(self._h, C.byref(n), C.byref(e)))
        return n.value, e.value

    # -- jx_insert
    def insert(self, vecs: torch.Tensor):
        assert vecs.dtype == _torch_dtype(self.dtype) and vecs.shape[1] == self.dim
        with torch.cuda.device(self.device):
            _check(_lib.jx_insert(self._h, _ptr(vecs), C.c_int64(vecs.shape[0]), _stream()))

    # -- jx_import_graph / jx_export_graph
    def import_graph(self, vecs, adj, entry):
        assert vecs.dtype == _torch_dtype(self.dtype)
        assert adj.dtype in (torch.int32, torch.uint32)
        assert adj.shape == (vecs.shape[0], self.R)
        with torch.cuda.device(self.device):
            _check(_lib.jx_import_graph(self._h, _ptr(vecs), C.c_int64(vecs.shape[0]), _ptr(adj), C.c_uint32(entry),
                                        _stream()))

    def export_graph(self):
        n, _ = self.size()
        adj = torch.empty((n, self.R), dtype=torch.int32, device=self.device)
        deg = torch.empty(n, dtype=torch.int32, device=self.device)
        with torch.cuda.device(self.device):
            _check(_lib.jx_export_graph(self._h, _ptr(adj), _ptr(deg), _stream()))
        return adj, deg

    # -- jx_quantize / jx_export_codes / stage entry points
    def quantize(self, bits, rotation, centroid=None, query_bits=8, rule=RULE_DEFAULT):
        assert rotation.dtype == torch.float32 and rotation.shape == (self.dim, self.dim)
        with torch.cuda.device(self.device):
            _check(_lib.jx_quantize(self._h, C.c_int32(bits), _ptr(rotation), _ptr(centroid), C.c_int32(query_bits),
                                    C.c_int32(rule), _stream()))
        self.bits = bits

    def import_codes(self, bits, rotation, centroid, codes, meta, query_bits=8):
        assert codes.dtype == torch.uint8 and meta.dtype == torch.float32
        with torch.cuda.device(self.device):
            _check(_lib.jx_import_codes(self._h, C.c_int32(bits), _ptr(rotation), _ptr(centroid), C.c_int32(query_bits),
                                        _ptr(codes), _ptr(meta), _stream()))
        self.bits = bits

    def export_codes(self):
        n, _ = self.size()
        codes = torch.empty((n, self.dim * self.bits // 8), dtype=torch.uint8, device=self.device)
        meta = torch.empty((n, 2), dtype=torch.float32, device=self.device)
        cen = torch.empty(self.dim, dtype=torch.float32, device=self.device)
        with torch.cuda.device(self.device):
            _check(_lib.jx_export_codes(self._h, _ptr(codes), _ptr(meta), _ptr(cen), _stream()))
        return codes, meta, cen

    def rotate(self, x):
        out = torch.empty_like(x)
        with torch.cuda.device(self.device):
            _check(_lib.jx_rotate(self._h, _ptr(x), C.c_int64(x.shape[0]), _ptr(out), _stream()))
        return out

    def rotate_points(self, x):
        assert x.dtype == _torch_dtype(self.dtype) and x.shape[1] == self.dim
        out = torch.empty(x.shape, dtype=torch.float32, device=self.device)
        with torch.cuda.device(self.device):
            _check(_lib.jx_rotate_points(self._h, _ptr(x), C.c_int64(x.shape[0]), _ptr(out), _stream()))
        return out

    def encode_rotated(self, r):
        n = r.shape[0]
        codes = torch.empty((n, self.dim * self.bits // 8), dtype=torch.uint8, device=self.device)
        meta = torch.empty((n, 2), dtype=torch.float32, device=self.device)
        with torch.cuda.device(self.device):
            _check(_lib.jx_encode_rotated(self._h, _ptr(r), C.c_int64(n), _ptr(codes), _ptr(meta), _stream()))
        return codes, meta

    # -- jx_search / jx_beam_frontier / jx_bruteforce
    def search(self, queries, k, L, mode=EXACT, rerank=0, stats=False, out=None):
        nq = queries.shape[0]
        if out is None:
            ids = torch.empty((nq, k), dtype=torch.int32, device=self.device)
            dist = torch.empty((nq, k), dtype=torch.float32, device=self.device)
        else:
            ids, dist = out
        st = Stats() if stats else None
        with torch.cuda.device(self.device):
            _check(_lib.jx_search(self._h, _ptr(queries), C.c_int64(nq), C.c_int32(k), C.c_int32(L), C.c_int32(mode),
                                  C.c_int32(rerank), _ptr(ids), _ptr(dist), C.byref(st) if stats else None, _stream()))
        return (ids, dist, st.as_dict()) if stats else (ids, dist)

    def beam_frontier(self, queries, L, mode=EXACT, stats=False):
        nq = queries.shape[0]
        ids = torch.empty((nq, L), dtype=torch.int32, device=self.device)
        dist = torch.empty((nq, L), dtype=torch.float32, device=self.device)
        st = Stats() if stats else None
        with torch.cuda.device(self.device):
            _check(_lib.jx_beam_frontier(self._h, _ptr(queries), C.c_int64(nq), C.c_int32(L), C.c_int32(mode),
                                         _ptr(ids), _ptr(dist), C.byref(st) if stats else None, _stream()))
        return (ids, dist, st.as_dict()) if stats else (ids, dist)

    def bruteforce(self, queries, k):
        nq = queries.shape[0]
        ids = torch.empty((nq, k), dtype=torch.int32, device=self.device)
        dist = torch.empty((nq, k), dtype=torch.float32, device=self.device)
        with torch.cuda.device(self.device):
            _check(_lib.jx_bruteforce(self._h, _ptr(queries), C.c_int64(nq), C.c_int32(k), _ptr(ids), _ptr(dist),
                                      _stream()))
        return ids, dist

    # -- jx_delete / jx_consolidate / jx_deleted_count
    def delete(self, ids: torch.Tensor):
        assert ids.dtype == torch.int32 and ids.dim() == 1
        with torch.cuda.device(self.device):
            _check(_lib.jx_delete(self._h, _ptr(ids), C.c_int64(ids.shape[0]), _stream()))

    def consolidate(self):
        with torch.cuda.device(self.device):
            _check(_lib.jx_consolidate(self._h, _stream()))

    def compact(self, want_map=True):
        """jx_compact; returns old id -> new id (int32 tensor, -1 = NONE for removed vertices) if asked."""
        n_old, _ = self.size()
        m = torch.empty(n_old, dtype=torch.int32, device=self.device) if want_map else None
        with torch.cuda.device(self.device):
            _check(_lib.jx_compact(self._h, _ptr(m), _stream()))
        return m

    def deleted_count(self):
        n = C.c_int64()
        with torch.cuda.device(self.device):
            _check(_lib.jx_deleted_count(self._h, C.byref(n), _stream()))
        return n.value


STATIC_SCRATCH_BYTES = 16 << 20


def bruteforce_static(base: torch.Tensor, queries: torch.Tensor, k: int, out=None):
    """jx_bruteforce_static: exhaustive kNN without an index or an arena; the caller passes the output tensors
    (`out`) when it must not allocate either."""
    dtype = {torch.uint8: U8, torch.float32: F32, torch.float16: F16}[base.dtype]
    assert queries.dtype == base.dtype and queries.shape[1] == base.shape[1]
    nq = queries.shape[0]
    if out is None:
        out = (torch.empty((nq, k), dtype=torch.int32, device=base.device),
               torch.empty((nq, k), dtype=torch.float32, device=base.device))
    ids, dist = out
    with torch.cuda.device(base.device):
        _check(_lib.jx_bruteforce_static(_ptr(base), C.c_int64(base.shape[0]), C.c_int32(base.shape[1]), C.c_int32(dtype),
                                         _ptr(queries), C.c_int64(nq), C.c_int32(k), _ptr(ids), _ptr(dist), _stream()))
    return ids, dist


def bruteforce_kernel() -> str:
    """jx_bruteforce_kernel: what the calling thread's last exhaustive search launched."""
    return _lib.jx_bruteforce_kernel().decode()


def mips_augment(x: torch.Tensor, max_norm: float = 0.0, is_query: bool = False, dim_out: int = 0, want_norms: bool = False):
    """jx_mips_augment.  Returns the augmented rows (if dim_out > 0) and / or the row norms."""
    assert x.dtype == torch.float32 and x.is_contiguous()
    n, dim = x.shape
    out = torch.empty((n, dim_out), dtype=torch.float32, device=x.device) if dim_out else None
    norms = torch.empty(n, dtype=torch.float32, device=x.device) if want_norms else None
    with torch.cuda.device(x.device):
        _check(_lib.jx_mips_augment(_ptr(x), C.c_int64(n), C.c_int32(dim), C.c_float(max_norm), C.c_int32(int(is_query)),
                                    _ptr(out), C.c_int32(dim_out), _ptr(norms), _stream()))
    if out is not None and norms is not None:
        return out, norms
    return out if out is not None else norms


def probe_gather(table: torch.Tensor, rec_bytes: int, ids: torch.Tensor, blocks: int = 4096):
    """jx_probe_gather: independent gathers of rec_bytes-byte records; returns the checksum words."""
    assert table.dtype == torch.uint8 and ids.dtype == torch.int32
    n_rec = table.numel() // rec_bytes
    assert 0 <= int(ids.min()) and int(ids.max()) < n_rec  # the device does not check
    sink = torch.empty(blocks * 256, dtype=torch.int32, device=table.device)
    with torch.cuda.device(table.device):
        _check(_lib.jx_probe_gather(_ptr(table), C.c_int64(n_rec), C.c_int32(rec_bytes), _ptr(ids), C.c_int64(ids.numel()),
                                    C.c_int32(blocks), _ptr(sink), _stream()))
    return sink


# -- attention beside the index: jx_kv_plan .. jx_found_attention.  These are called many times in each step of a model, over
# operands of a few microseconds' work: their checks are written to be quick.  They are a serving program's: inputs that require a gradient
# are refused unless gradients are switched off.

_HEAD_TYPES = {torch.float16: F16, torch.bfloat16: BF16}
_I32, _I64, _F32 = torch.int32, torch.int64, torch.float32


def _run(fn, i, *args):
    """Calls an entry point with the current stream of GPU i as its last argument."""
    if torch.cuda.current_device() == i:
        rc = fn(*args, _raw_stream(i))
    else:
        with torch.cuda.device(i):
            rc = fn(*args, _raw_stream(i))
    if rc:
        _check(rc)


def _gpu(t):
    """The GPU of a call's first tensor; all the others have to be there too."""
    i = t.get_device()
    assert i >= 0, "not on a GPU"
    return i


def _no_gradient(t):
    assert not (t.requires_grad and torch.is_grad_enabled()), "no gradient goes through the attention calls: make them under torch.no_grad()"


def _rows(t, i, dtype):
    """A tensor of any strides whose last dimension holds a head's elements."""
    _no_gradient(t)
    assert t.get_device() == i and t.dtype is dtype and (t.stride(-1) == 1 or t.shape[-1] == 1), (t.device, i, t.dtype)
    return t.data_ptr()


def _array(t, i, dtype, *shape):
    assert t.get_device() == i and t.is_contiguous() and t.dtype is dtype and t.shape == shape, (t.device, i, t.dtype, tuple(t.shape), shape)
    return t.data_ptr()


def _real(t, i, dtype, *shape):
    """An array that a model may have learnt or made."""
    _no_gradient(t)
    return _array(t, i, dtype, *shape)


def _alike(a, b):
    """Whether two tensors are laid out alike; the stride of a dimension of one has no meaning."""
    if a.shape != b.shape:
        return False
    sa, sb = a.stride(), b.stride()
    return sa == sb or all(n <= 1 or x == y for n, x, y in zip(a.shape, sa, sb))


def _kv_cache(k_cache, v_cache, i, dtype, head_dim):
    pages, page, _, d = k_cache.shape
    strides = k_cache.stride()
    assert d == head_dim and _alike(k_cache, v_cache)
    return KvCache(_rows(k_cache, i, dtype), _rows(v_cache, i, dtype), strides[0], strides[1], strides[2], page, pages)


def kv_plan(lens, new, table, free, n_free, page, n_tokens, out=None) -> KvPlan:
    """jx_kv_plan: `table` gets the new pages in place; `n_free` stays, the number left is in the result.  n_tokens: rows of the
    step (the host's bound on the sum of `new`).  `out`: a KvPlan to write into."""
    n, w, f = lens.shape[0], table.shape[1], free.shape[0]
    i = _gpu(lens)
    if out is None:
        # the 64-bit slots first, then the 32-bit arrays, in one allocation
        block = torch.empty(3 * n_tokens + 2 * n + 2, dtype=_I32, device=lens.device)
        slot, pos, q_start, kv_len, left = block.split((2 * n_tokens, n_tokens, n + 1, n, 1))
        out = KvPlan(q_start, kv_len, pos, slot.view(_I64), left)
        p_slot = block.data_ptr()
        p_pos = p_slot + 8 * n_tokens
        p_start = p_pos + 4 * n_tokens
        p_len = p_start + 4 * (n + 1)
        p_left = p_len + 4 * n
    else:
        p_left, p_start, p_len = _array(out.n_free, i, _I32, 1), _array(out.q_start, i, _I32, n + 1), _array(out.kv_len, i, _I32, n)
        p_pos, p_slot = _array(out.pos, i, _I32, n_tokens), _array(out.slot, i, _I64, n_tokens)
    _run(_lib.jx_kv_plan, i, _array(lens, i, _I32, n), _array(new, i, _I32, n), n, page, _array(table, i, _I32, n, w), w,
         _array(free, i, _I32, f), _array(n_free, i, _I32, 1), f, p_left, p_start, p_len, p_pos, p_slot, n_tokens)
    return out


def kv_release(first, end, table, free, n_free):
    """jx_kv_release: pages first[r] .. end[r] - 1 of row r go back; `table`, `free` and `n_free` are updated in place."""
    n, w, f = first.shape[0], table.shape[1], free.shape[0]
    i = _gpu(table)
    _run(_lib.jx_kv_release, i, _array(first, i, _I32, n), _array(end, i, _I32, n), n, _array(table, i, _I32, n, w), w,
         _array(free, i, _I32, f), _array(n_free, i, _I32, 1), f)


def qk_norm_rope(q, k, v, k_cache, v_cache, pos, slot, cos=None, sin=None, q_weight=None, k_weight=None, eps=1e-6, interleaved=False,
                 out=None):
    """jx_qk_norm_rope: the queries [tokens][heads][head_dim] made ready (in `out`, which may be a contiguous q); keys and values
    go to their slots of the caches [pages][page][kv_heads][head_dim] (any strides, alike in both)."""
    t, h, d = q.shape
    kv = k_cache.shape[2]
    dt, i = q.dtype, _gpu(q)
    if out is None:
        out = torch.empty((t, h, d), dtype=dt, device=q.device)
    else:
        _array(out, i, dt, t, h, d)
    n_pos, half = cos.shape if cos is not None else (0x7FFFFFFF, 0)
    assert k.shape == v.shape == (t, kv, d)
    qs, ks, vs = q.stride(), k.stride(), v.stride()
    a = RopeArgs(_HEAD_TYPES[dt], h, kv, d, 2 * half, interleaved, t, n_pos, _rows(q, i, dt), _rows(k, i, dt), _rows(v, i, dt), qs[0], qs[1], ks[0],
                 ks[1], vs[0], vs[1], _real(q_weight, i, dt, d) if q_weight is not None else None,
                 _real(k_weight, i, dt, d) if k_weight is not None else None, eps, _real(cos, i, _F32, n_pos, half) if half else None,
                 _real(sin, i, _F32, n_pos, half) if half else None, _array(pos, i, _I32, t), _array(slot, i, _I64, t), out.data_ptr(),
                 _kv_cache(k_cache, v_cache, i, dt, d))
    _run(_lib.jx_qk_norm_rope, i, C.byref(a))
    return out


def _outputs(out, q, i, t, h, d):
    """The pair to write into, made here if there is none, and its pointers."""
    if out is None:
        o, lse = torch.empty((t, h, d), dtype=q.dtype, device=q.device), torch.empty((t, h), dtype=_F32, device=q.device)
        return o, lse, o.data_ptr(), lse.data_ptr()
    o, lse = out
    return o, lse, _array(o, i, q.dtype, t, h, d), _array(lse, i, _F32, t, h) if lse is not None else None


def paged_attention(q, k_cache, v_cache, table, q_start, kv_len, scale, window=0, out=None, work=None):
    """jx_paged_attention: (out [tokens][heads][head_dim], lse [tokens][heads]).  `out`: those two, to write into (lse may be None);
    `work`: a uint8 tensor as large as the call needs (made here where it is None)."""
    t, h, d = q.shape
    n, w = table.shape
    dt, i = q.dtype, _gpu(q)
    o, lse, p_out, p_lse = _outputs(out, q, i, t, h, d)
    qs = q.stride()
    a = AttendArgs(_HEAD_TYPES[dt], h, k_cache.shape[2], d, t, _rows(q, i, dt), qs[0], qs[1], _kv_cache(k_cache, v_cache, i, dt, d),
                   _array(table, i, _I32, n, w), w, n, _array(q_start, i, _I32, n + 1), _array(kv_len, i, _I32, n), scale, window, p_out, p_lse)
    ref = C.byref(a)
    if work is None:
        nbytes = _lib.jx_paged_attention_bytes(ref)
        if nbytes < 0:
            _check(int(nbytes))
        work = torch.empty(nbytes, dtype=torch.uint8, device=q.device)
    else:
        nbytes = work.shape[0]
        _array(work, i, torch.uint8, nbytes)
    _run(_lib.jx_paged_attention, i, ref, work.data_ptr(), nbytes)
    return o, lse


def found_attention(q, keys, values, ids, scale, part=None, out=None):
    """jx_found_attention: (out, lse) over the rows ids [tokens][heads][k] of keys and values [rows][kv_heads][head_dim] (any
    strides, alike in both), joined with part = (out, lse) of other keys if given.  `out`: two tensors to write into (may be `part`)."""
    t, h, d = q.shape
    n, kv, kd = keys.shape
    k = ids.shape[2]
    dt, i = q.dtype, _gpu(q)
    o, lse, p_out, p_lse = _outputs(out, q, i, t, h, d)
    qs, ks = q.stride(), keys.stride()
    assert kd == d and _alike(keys, values)
    a = FoundArgs(_HEAD_TYPES[dt], h, kv, d, t, _rows(q, i, dt), qs[0], qs[1], _rows(keys, i, dt), _rows(values, i, dt), ks[0], ks[1], n,
                  _array(ids, i, _I32, t, h, k), k, scale, _real(part[0], i, dt, t, h, d) if part else None,
                  _real(part[1], i, _F32, t, h) if part else None, p_out, p_lse)
    _run(_lib.jx_found_attention, i, C.byref(a))
    return o, lse


def ids_to_numpy(t: torch.Tensor):
    """int32 device tensor of ids -> uint32 numpy array."""
    import numpy as np

    return t.cpu().numpy().view(np.uint32)
