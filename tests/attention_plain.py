"""Attention beside the index from its definitions, in 64 bits on the CPU, one row at a time, with bounds on what the kernels'
roundings may change.

Bounds.  u is the unit roundoff of the element type (2^-8 bfloat16, 2^-11 binary16), tiny its smallest step (subnormal).  With weights
w_j (sum 1) and A = sum_j w_j |v_j|, per element:
  scores      float32 products summed in any order: an error of at most d_s = (dim + 4) 2^-24 scale max_j sum_e |q_e k_je| each, which
              changes a weight by a factor within 1 +- 2 d_s, the output by at most 4 d_s A (numerator and denominator)
  weights     rounded to the element type: u A, and half a smallest step of that type for each key relative to the largest weight,
              of which the sum is at least one: tiny / 2 sum_j |v_j|
  sums        n keys added in float32, some of them rescaled: 2 (n + 64) 2^-24 A, exponentials within 2^-22: 2^-21 A
  result      rounded once: u |out| + tiny / 2
The log-sum-exp: d_s + (n + 64) 2^-24 + 2^-21 + 2^-22 |lse|.
"""
import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


def attend_row(q, k, v, scale, dtype, rounded=True):
    """(out, lse, bound of out, bound of lse) of one query row over the keys it sees, everything float64."""
    dim, n = q.shape[0], k.shape[0]
    if n == 0:
        z = torch.zeros(dim, dtype=torch.float64)
        return z, -math.inf, z, 0.0
    s = (k @ q) * scale
    d_s = (dim + 4) * 2.0 ** -24 * abs(scale) * float((k.abs() @ q.abs()).max())
    lse = torch.logsumexp(s, 0)
    w = torch.exp(s - lse)
    out, a = w @ v, w @ v.abs()
    u, tiny = UNIT[dtype], TINY[dtype]
    bound = (4 * d_s + 2 * (n + 64) * 2.0 ** -24 + 2.0 ** -21) * a + u * out.abs() + tiny / 2
    if rounded:
        bound = bound + u * a + tiny / 2 * v.abs().sum(0)
    return out, float(lse), bound * 1.02, d_s + (n + 64) * 2.0 ** -24 + 2.0 ** -21 + 2.0 ** -22 * abs(float(lse))


def seen_keys(table_row, kv_len, n, i, page, n_pages, window):
    """(page, place) of every key that row i of the last n sees."""
    p = kv_len - n + i
    lo = max(0, p - window + 1) if window else 0
    out = []
    for j in range(lo, p + 1):
        if j // page >= len(table_row):
            break
        at = int(table_row[j // page])
        if 0 <= at < n_pages:
            out.append((at, j % page))
    return out


def paged(q, k_cache, v_cache, table, q_start, kv_len, scale, window, rows=None):
    """{(t, h): attend_row(...)} for all rows, or those of `rows`."""
    dtype = q.dtype
    q, k_cache, v_cache = q.cpu().double(), k_cache.cpu(), v_cache.cpu()
    t_n, h_n, dim = q.shape
    pages, page, kv, _ = k_cache.shape
    table, q_start, kv_len = table.cpu().tolist(), q_start.cpu().tolist(), kv_len.cpu().tolist()
    res = {}
    for t in range(t_n):
        if rows is not None and t not in rows:
            continue
        keys = []
        for r in range(len(kv_len)):
            if q_start[r] <= t < q_start[r + 1]:
                keys = seen_keys(table[r], kv_len[r], q_start[r + 1] - q_start[r], t - q_start[r], page, pages, window)
        at = torch.tensor(keys, dtype=torch.int64).reshape(-1, 2)
        for h in range(h_n):
            c = h // (h_n // kv)
            res[t, h] = attend_row(q[t, h], k_cache[at[:, 0], at[:, 1], c].double(), v_cache[at[:, 0], at[:, 1], c].double(), scale, dtype)
    return res


def found(q, keys, values, ids, scale, part=None):
    dtype = q.dtype
    q, keys, values, ids = q.cpu().double(), keys.cpu(), values.cpu(), ids.cpu().long()
    t_n, h_n, dim = q.shape
    n, kv, _ = keys.shape
    res = {}
    for t in range(t_n):
        for h in range(h_n):
            i = ids[t, h]
            i = i[(i >= 0) & (i < n)]
            c = h // (h_n // kv)
            out, lse, bo, bl = attend_row(q[t, h], keys[i, c].double(), values[i, c].double(), scale, dtype, rounded=False)
            if part is not None and part[1][t, h] != -math.inf:
                po, pl = part[0][t, h].cpu().double(), float(part[1][t, h])
                top = max(lse, pl)
                a, b = math.exp(lse - top), math.exp(pl - top)
                # the list's share is off by as much as its own result and weight are, the part's weight by float32's step at |lse|
                da = bl + 2.0 ** -22 * (abs(pl) + abs(lse) if len(i) else abs(pl))
                bo = (a * (bo + da * out.abs()) + b * da * po.abs()) / (a + b) + UNIT[dtype] * (out.abs() * a + po.abs() * b) / (a + b) + \
                    da * (out.abs() * a + po.abs() * b) / (a + b) + TINY[dtype]
                out, lse = (a * out + b * po) / (a + b), top + math.log(a + b)
                bl = bl + da + 2.0 ** -21 + 2.0 ** -22 * abs(lse)
            res[t, h] = out, lse, bo, bl
    return res


def check(got, want, what=""):
    out, lse = got[0].cpu().double(), got[1].cpu().double()
    for (t, h), (o, l, bo, bl) in want.items():
        err = (out[t, h] - o).abs()
        assert bool((err <= bo).all()), (what, t, h, "out", float((err - bo).max()), float(err.max()))
        if l == -math.inf:
            assert float(lse[t, h]) == -math.inf and not out[t, h].any(), (what, t, h, float(lse[t, h]))
        else:
            assert abs(float(lse[t, h]) - l) <= bl, (what, t, h, "lse", float(lse[t, h]), l, bl)
