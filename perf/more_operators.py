"""Measured cases of the operators over a cache of 8 bits.

Keys and values are held as e4m3, with one power of two (e8m0) for each block of tokens and key head:

  store   queries and keys normalised per head and rotated, keys and values put into their blocks in 8 bits; a block whose scale
          grows has what it already holds brought to the new one
  attend  attention of the new tokens over the paged cache of 8 bits
  found   attention of every (token, head) over rows of 8 bits that its search returned, joined with what `attend` gave

Queries and keys have unit mean square, as the norm leaves them, the queries with a gain; the size of values differs from block to
block; pages are scattered over the cache; lengths spread over a factor of sixteen under the longest.
"""
import math
import random

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
CODE, SCALE = torch.float8_e4m3fn, torch.float8_e8m0fnu
BASE = 10000.0
EPS = 1e-6
GAIN = 1.5


def listed():
    return [
        # a decode step: a token each, somewhere in a block that holds others already
        _store("store_step", "bf16", tokens=64, requests=64, heads=32, kv_heads=8, dim=128, rot=128, page=16, block=16, pairs=False),
        # a prompt's chunk, an odd number of tokens, half of each head rotated, neighbours as pairs
        _store("store_chunk", "f16", tokens=8191, requests=1, heads=32, kv_heads=8, dim=128, rot=64, page=64, block=32, pairs=True),
        # many requests of unlike numbers of tokens, long heads, a scale for every token
        _store("store_mixed", "bf16", tokens=1111, requests=150, heads=16, kv_heads=2, dim=256, rot=128, page=16, block=1, pairs=False),
        # one user, a short context: latency
        _attend("attend_one_short", "bf16", requests=1, chunk=1, longest=777, heads=32, kv_heads=8, dim=128, page=16, block=16),
        # a decode step of an ordinary batch
        _attend("attend_step", "bf16", requests=64, chunk=1, longest=8192, heads=32, kv_heads=8, dim=128, page=16, block=16),
        # few users, very long contexts of unlike lengths
        _attend("attend_step_long", "f16", requests=4, chunk=1, longest=131072, heads=64, kv_heads=8, dim=128, page=64, block=64),
        # a prompt's last chunk over what is in the cache
        _attend("attend_prompt", "bf16", requests=1, chunk=4096, longest=16384, heads=32, kv_heads=8, dim=128, page=64, block=32),
        # decode steps and chunks mixed, as many key heads as query heads, a sliding window
        _attend("attend_mixed_window", "f16", requests=33, chunk=509, longest=8000, heads=16, kv_heads=16, dim=64, page=8, block=4, window=1024),
        # long heads, one key head for all
        _attend("attend_wide_heads", "bf16", requests=9, chunk=301, longest=4001, heads=8, kv_heads=1, dim=256, page=32, block=16),
        # ten neighbours for each head of a decode step
        _found("found_step", "bf16", tokens=16, heads=32, kv_heads=8, dim=128, k=10, rows=100_000, block=16),
        # a chunk of a prompt, a hundred neighbours for each head
        _found("found_chunk", "f16", tokens=1000, heads=32, kv_heads=8, dim=128, k=100, rows=1_000_000, block=64),
    ]


def _store(name, dtype, tokens, requests, heads, kv_heads, dim, rot, page, block, pairs):
    return dict(name=name, op="store", dtype=dtype, tokens=tokens, requests=requests, heads=heads, kv_heads=kv_heads, dim=dim, rot=rot,
                page=page, block=block, pairs=pairs)


def _attend(name, dtype, requests, chunk, longest, heads, kv_heads, dim, page, block, window=0):
    return dict(name=name, op="attend", dtype=dtype, requests=requests, chunk=chunk, longest=longest, heads=heads, kv_heads=kv_heads,
                dim=dim, page=page, block=block, window=window)


def _found(name, dtype, tokens, heads, kv_heads, dim, k, rows, block):
    return dict(name=name, op="found", dtype=dtype, tokens=tokens, heads=heads, kv_heads=kv_heads, dim=dim, k=k, rows=rows, block=block)


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    top = [work(c) for c in listed()]
    flops, size = max(w["flops"] for w in top), max(w["bytes"] for w in top)
    while True:
        op = rng.choice(["store", "attend", "attend", "attend", "found"])
        dtype = rng.choice(["bf16", "f16"])
        dim = rng.choice([64, 80, 96, 128, 128, 128, 192, 256])
        kv_heads = rng.choice([1, 2, 4, 8, 16])
        heads = kv_heads * rng.choice([1, 2, 3, 4, 6, 8])
        page = rng.choice([8, 16, 16, 32, 64, 128])
        block = rng.choice([b for b in (1, 2, 4, 8, 16, 16, 32, 64) if b <= page])
        if op == "store":
            rot = rng.choice([r for r in (32, 64, 96, 128) if r <= dim])
            tokens = log(1, 8191)
            c = _store("", dtype, tokens, log(1, tokens), heads, kv_heads, dim, rot, page, block, rng.random() < 0.5)
            # the plain form holds a whole block for each token
            if tokens * block * kv_heads * dim > 2 ** 28:
                continue
        elif op == "attend":
            longest = log(16, 131072)
            chunk = 1 if rng.random() < 0.4 else log(1, min(4096, longest))
            c = _attend("", dtype, log(1, 200), chunk, longest, heads, kv_heads, dim, page, block, rng.choice([0, 0, 0, log(16, 4096)]))
            reqs = _lengths(c)
            # the plain form holds the keys of all single tokens, or the scores of one request's heads, at once
            if sum(n for _, n in reqs) > 16384 or max(n * L for L, n in reqs) * heads > 2 ** 31 or \
                    (chunk == 1 and longest * len(reqs) * kv_heads * dim > 2 ** 31):
                continue
        else:
            c = _found("", dtype, log(1, 1000), heads, kv_heads, dim, log(1, 128), log(1000, 1_000_000), block)
            if c["rows"] * kv_heads * dim > 2 ** 30 or c["tokens"] * heads * c["k"] * dim > 2 ** 29:
                continue
        w = work(c)
        if w["flops"] <= flops and w["bytes"] <= size:
            return c


def _lengths(case):
    """(length in the cache with the new tokens, new tokens) of every request; the first has the longest of both."""
    rng = random.Random("lengths of %d requests up to %d, %d" % (case["requests"], case["longest"], case["chunk"]))
    out = [(case["longest"], min(case["chunk"], case["longest"]))]
    for _ in range(case["requests"] - 1):
        L = int(round(case["longest"] * 16 ** -rng.random()))
        n = int(round(case["chunk"] ** rng.random()))
        out.append((max(L, 1), max(1, min(n, L))))
    rng.shuffle(out)
    return out


def _spans(case):
    """(position of the first new token, new tokens) of every request of a `store` case; together a little less than the rows of the
    step where that is large: the rest is padding."""
    rng = random.Random("spans of %d tokens in %d requests" % (case["tokens"], case["requests"]))
    used = case["tokens"] - case["tokens"] // 100
    n = min(case["requests"], used)
    cuts = sorted(rng.sample(range(1, used), n - 1)) if n > 1 else []
    return [(rng.randrange(0, 24000), b - a) for a, b in zip([0] + cuts, cuts + [used])]


def _pairs(L, n, window):
    """(query, key) pairs of a request whose last n of L positions ask."""
    if not window:
        return n * (L - n) + n * (n + 1) // 2
    return sum(min(window, p + 1) for p in range(L - n, L))


def work(case):
    h, kv, d, block = case["heads"], case["kv_heads"], case["dim"], case["block"]
    if case["op"] == "store":
        t = case["tokens"]
        blocks = min(t, -(-t // block) + case["requests"])
        return {"bytes": t * (h * d * 4 + 2 * kv * d * 3 + case["rot"] * 4 + 12) + blocks * kv * 2, "flops": t * (h + kv) * (4 * d + 3 * case["rot"]) + t * 4 * kv * d}
    if case["op"] == "attend":
        size = flops = 0
        for L, n in _lengths(case):
            first = max(0, L - n + 1 - case["window"]) if case["window"] else 0
            size += n * h * (4 * d + 4) + (L - first) * kv * d * 2 + -(-(L - first) // block) * kv * 2 + -(-(L - first) // case["page"]) * 4 + 8
            flops += 4 * d * h * _pairs(L, n, case["window"])
        return {"bytes": size, "flops": flops}
    lists, held = case["tokens"] * h, case["rows"] * kv
    rows = held * -math.expm1(-lists * case["k"] / held)  # so many different ones are asked for
    return {"bytes": int(rows * (2 * d + 2 / block)) + lists * (case["k"] * 4 + 6 * d + 8), "flops": lists * case["k"] * 4 * d}


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(g, shape, dtype, gain=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(gain).to(dtype)


def _exponents(largest):
    """The scale's byte for blocks whose largest value has this size: codes of 128 up to 256."""
    return ((largest.view(torch.int32) >> 23) - 7).clamp(min=1)


def _power(byte):
    """2^(byte - 127) of bytes 1 .. 254, in 32 bits."""
    return (byte.to(torch.int32) << 23).view(torch.float32)


def _blocks(g, n, block, kv, d, spread):
    """Codes [n][block][kv][d] and scales [n][kv] of blocks of normal values of unlike size, made in parts."""
    codes = torch.empty((n, block, kv, d), dtype=CODE, device="cuda")
    scales = torch.empty((n, kv), dtype=SCALE, device="cuda")
    step = max(1, (1 << 26) // (block * kv * d))
    for a in range(0, n, step):
        b = slice(a, min(n, a + step))
        x = torch.randn((b.stop - a, block, kv, d), generator=g, device="cuda")
        x *= torch.exp(spread * torch.randn((b.stop - a, 1, kv, 1), generator=g, device="cuda"))
        byte = _exponents(x.abs().amax((1, 3)))
        codes[b] = (x * _power(254 - byte)[:, None, :, None]).to(CODE)
        scales.view(torch.uint8)[b] = byte.to(torch.uint8)
    return codes, scales


def _cache(g, pages, page, block, kv, d, spread):
    """A cache's pages [pages][page][kv][d] and scales [pages][page / block][kv]."""
    codes, scales = _blocks(g, pages * (page // block), block, kv, d, spread)
    return codes.view(pages, page, kv, d), scales.view(pages, page // block, kv)


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device="cuda")


def prepare(case, seed):
    g = _generator(seed)
    dtype, h, kv, d, block = TYPES[case["dtype"]], case["heads"], case["kv_heads"], case["dim"], case["block"]
    st = {"case": dict(case), "block": block, "scale": d ** -0.5}
    if case["op"] == "store":
        t, page = case["tokens"], case["page"]
        spans = _spans(case)
        first, count = (np.array(x, dtype=np.int64) for x in zip(*spans))
        used = int(count.sum())
        of = np.repeat(np.arange(len(count)), count)
        position = first[of] + np.arange(used) - (np.cumsum(count) - count)[of]
        held = (first + count - 1) // page - first // page + 1  # pages that the new tokens of a request lie in
        before = np.cumsum(held) - held
        pages = int(held.sum()) + 9
        order = torch.randperm(pages, generator=g, device="cuda")
        at = _ints((before[of] + position // page - first[of] // page).tolist(), torch.int64)
        place = _ints((position % page).tolist(), torch.int64)
        pos = torch.full((t,), -1, dtype=torch.int32, device="cuda")
        slot = torch.full((t,), -1, dtype=torch.int64, device="cuda")
        pos[:used] = _ints(position.tolist())
        slot[:used] = order[at] * page + place
        fused = _normal(g, (t, (h + 2 * kv) * d), dtype, 2.0)  # one projection's output
        q, k, v = (x.unflatten(1, (-1, d)) for x in fused.split([h * d, kv * d, kv * d], 1))
        angle = torch.arange(32768, device="cuda", dtype=torch.float64)[:, None] * \
            BASE ** (-torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / case["rot"])
        k_cache, k_scale = _cache(g, pages, page, block, kv, d, 0.2)
        v_cache, v_scale = _cache(g, pages, page, block, kv, d, 0.7)
        st.update(q=q, k=k, v=v, pos=pos, slot=slot, used=used, cos=angle.cos().float(), sin=angle.sin().float(), pairs=case["pairs"],
                  k_cache=k_cache, v_cache=v_cache, k_scale=k_scale, v_scale=v_scale,
                  q_weight=_normal(g, (d,), dtype, 0.1) + 1, k_weight=_normal(g, (d,), dtype, 0.1) + 1)
        return st
    if case["op"] == "attend":
        reqs, page = _lengths(case), case["page"]
        held = [-(-L // page) for L, _ in reqs]
        pages = sum(held) + max(held) // 8 + 1
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        width = max(held) * 5 // 4 + 1
        table = torch.full((len(reqs), width), -1, dtype=torch.int32, device="cuda")
        start = _ints([0] + list(np.cumsum(held)), torch.int64)
        at = torch.arange(width, device="cuda")[None, :]
        mask = at < _ints(held, torch.int64)[:, None]
        table[mask] = order[(start[:-1, None] + at)[mask]]
        k_cache, k_scale = _cache(g, pages, page, block, kv, d, 0.2)
        v_cache, v_scale = _cache(g, pages, page, block, kv, d, 0.7)
        st.update(q=_normal(g, (sum(n for _, n in reqs), h, d), dtype, GAIN), k_cache=k_cache, v_cache=v_cache, k_scale=k_scale,
                  v_scale=v_scale, table=table, q_start=_ints([0] + list(np.cumsum([n for _, n in reqs]))),
                  kv_len=_ints([L for L, _ in reqs]), reqs=reqs, window=case["window"])
        return st
    t, k, rows = case["tokens"], case["k"], case["rows"]
    ids = torch.randint(0, rows, (t, h, k), generator=g, device="cuda", dtype=torch.int32)
    short = torch.rand((t, h, 1), generator=g, device="cuda") < 0.05  # a search that found fewer than it was asked for
    ids[short & (torch.arange(k, device="cuda") >= (k + 1) // 2)] = -1
    blocks = -(-rows // block)
    keys, k_scale = _blocks(g, blocks, block, kv, d, 0.2)
    values, v_scale = _blocks(g, blocks, block, kv, d, 0.7)
    st.update(q=_normal(g, (t, h, d), dtype, GAIN), keys=keys.flatten(0, 1)[:rows], values=values.flatten(0, 1)[:rows], k_scale=k_scale,
              v_scale=v_scale, ids=ids, out=_normal(g, (t, h, d), dtype, 0.2), lse=torch.randn((t, h), generator=g, device="cuda") + math.log(k) + 1)
    return st


def run(st):
    return (_own if own else _plain)[st["case"]["op"]](st)


# ---- the framework's calls ---------------------------------------------------------------------------------------------

def _own_store(st):
    from paper_2601_07048_amd import jx

    q = jx.qk_norm_rope8(st["q"], st["k"], st["v"], st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"], st["pos"], st["slot"],
                         st["cos"], st["sin"], q_weight=st["q_weight"], k_weight=st["k_weight"], eps=EPS, interleaved=st["pairs"])
    return {"q": q, "k_cache": st["k_cache"], "v_cache": st["v_cache"], "k_scale": st["k_scale"], "v_scale": st["v_scale"]}


def _own_attend(st):
    from paper_2601_07048_amd import jx

    out, lse = jx.paged_attention8(st["q"], st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"], st["table"], st["q_start"],
                                   st["kv_len"], st["scale"], window=st["window"])
    return {"out": out, "lse": lse}


def _own_found(st):
    from paper_2601_07048_amd import jx

    out, lse = jx.found_attention8(st["q"], st["keys"], st["values"], st["k_scale"], st["v_scale"], st["ids"], st["scale"], st["block"],
                                   part=(st["out"], st["lse"]))
    return {"out": out, "lse": lse}


_own = {"store": _own_store, "attend": _own_attend, "found": _own_found}


# ---- the plain forms ---------------------------------------------------------------------------------------------------

def _turn(x, weight, cos, sin, pairs):
    x = x.float()
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    half = cos.shape[-1]
    cos, sin = cos[:, None, :], sin[:, None, :]
    head, tail = x[..., :2 * half], x[..., 2 * half:]
    a, b = (head[..., 0::2], head[..., 1::2]) if pairs else (head[..., :half], head[..., half:])
    a, b = a * cos - b * sin, b * cos + a * sin
    head = torch.stack([a, b], -1).flatten(-2) if pairs else torch.cat([a, b], -1)
    return torch.cat([head, tail], -1)


def _put(x, cache, scale, slot, block):
    """Rows x [n][kv][d] into their slots."""
    kv, d = x.shape[1:]
    codes, byte = cache.view(-1, block, kv, d), scale.view(torch.uint8).view(-1, kv)
    at, place = slot // block, slot % block
    first = torch.full((len(codes),), block, dtype=torch.int64, device=x.device).scatter_reduce_(0, at, place, "amin")[at]
    largest = torch.zeros((len(codes), kv), device=x.device).scatter_reduce_(0, at[:, None].expand(-1, kv), x.abs().amax(-1), "amax")[at]
    old = byte[at].int()
    new = torch.maximum(_exponents(largest), torch.where(first[:, None] > 0, old, torch.zeros_like(old)))
    # what the block holds in front of its new tokens; every token of a block writes the same
    held = torch.arange(block, device=x.device)[None, :] < first[:, None]
    was = codes.view(torch.uint8)[at]
    less = _power(127 + (old - new).clamp(-126, 0))[:, None, :, None]
    now = (was.view(CODE).float() * less).to(CODE).view(torch.uint8)
    codes.view(torch.uint8)[at] = torch.where(held[:, :, None, None], now, was)
    codes.view(torch.uint8)[at, place] = (x * _power(254 - new)[..., None]).to(CODE).view(torch.uint8)
    byte[at] = new.to(torch.uint8)


def _plain_store(st):
    n, dtype = st["used"], st["q"].dtype
    cos, sin = st["cos"][st["pos"][:n].long()], st["sin"][st["pos"][:n].long()]
    q = torch.zeros(st["q"].shape, dtype=dtype, device=st["q"].device)
    q[:n] = _turn(st["q"][:n], st["q_weight"], cos, sin, st["pairs"]).to(dtype)
    _put(_turn(st["k"][:n], st["k_weight"], cos, sin, st["pairs"]), st["k_cache"], st["k_scale"], st["slot"][:n], st["block"])
    _put(st["v"][:n].float(), st["v_cache"], st["v_scale"], st["slot"][:n], st["block"])
    return {"q": q, "k_cache": st["k_cache"], "v_cache": st["v_cache"], "k_scale": st["k_scale"], "v_scale": st["v_scale"]}


def _pages(cache, scale, pages, block):
    """Values [..., tokens][kv][d] of the pages that a table names."""
    codes = cache.view(torch.uint8)[pages].view(CODE).float().unflatten(-3, (-1, block))
    return (codes * scale.view(torch.uint8)[pages].view(SCALE).float()[..., None, :, None]).flatten(-5, -3)


def _over(q, k, v, hidden, scale):
    """(out, lse) of queries [..., kv, rows, d] over keys [..., kv, L, d]."""
    s = torch.matmul(q * scale, k.transpose(-1, -2)).masked_fill_(hidden, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s.sub_(m))
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / total, (m + torch.log(total))[..., 0]


def _plain_attend(st):
    q, block, window = st["q"], st["block"], st["window"]
    t, h, d = q.shape
    page, kv = st["k_cache"].shape[1:3]
    if len(st["reqs"]) == t:  # a token each: all at once, up to the longest
        longest = max(L for L, _ in st["reqs"])
        pages = st["table"][:, :-(-longest // page)].clamp(min=0).long()
        k, v = (_pages(st[x + "_cache"], st[x + "_scale"], pages, block).transpose(1, 2) for x in "kv")
        j, last = torch.arange(k.shape[2], device=q.device), st["kv_len"].long()[:, None] - 1
        hidden = (j > last) | (j <= last - window) if window else j > last
        out, lse = _over(q.float().view(t, kv, h // kv, d), k, v, hidden[:, None, None, :], st["scale"])
        return {"out": out.reshape(t, h, d).to(q.dtype), "lse": lse.reshape(t, h)}
    out = torch.empty((t, h, d), dtype=torch.float32, device=q.device)
    lse = torch.empty((t, h), dtype=torch.float32, device=q.device)
    at = 0
    for r, (L, n) in enumerate(st["reqs"]):
        first = (max(0, L - n + 1 - window) if window else 0) // page
        pages = st["table"][r, first:-(-L // page)].long()
        k, v = (_pages(st[x + "_cache"], st[x + "_scale"], pages, block)[:L - first * page].transpose(0, 1) for x in "kv")
        i = torch.arange(L - n, L, device=q.device).repeat_interleave(h // kv)[:, None]
        j = torch.arange(first * page, L, device=q.device)[None, :]
        hidden = (j > i) | (j <= i - window) if window else j > i
        x = q[at:at + n].float().view(n, kv, h // kv, d).transpose(0, 1).reshape(kv, -1, d)
        o, w = _over(x, k, v, hidden, st["scale"])
        out[at:at + n] = o.view(kv, n, h // kv, d).transpose(0, 1).reshape(n, h, d)
        lse[at:at + n] = w.view(kv, n, h // kv).transpose(0, 1).reshape(n, h)
        at += n
    return {"out": out.to(q.dtype), "lse": lse}


def _plain_found(st):
    q, block = st["q"].float(), st["block"]
    h, d = q.shape[1:]
    ids = st["ids"].long()
    at = ids.clamp(min=0)
    head = (torch.arange(h, device=q.device) // (h // st["keys"].shape[1]))[None, :, None]

    def rows(codes, scale):
        return codes.view(torch.uint8)[at, head].view(CODE).float() * scale.view(torch.uint8)[at // block, head].view(SCALE).float()[..., None]

    s = (rows(st["keys"], st["k_scale"]) * q[:, :, None, :]).sum(-1) * st["scale"]
    s = s.masked_fill(ids < 0, -math.inf)
    m = torch.maximum(s.amax(-1), st["lse"])
    p, before = torch.exp(s - m[..., None]), torch.exp(st["lse"] - m)
    total = p.sum(-1) + before
    out = (p[..., None] * rows(st["values"], st["v_scale"])).sum(2) + before[..., None] * st["out"].float()
    return {"out": (out / total[..., None]).to(st["q"].dtype), "lse": m + torch.log(total)}


_plain = {"store": _plain_store, "attend": _plain_attend, "found": _plain_found}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    return {"store": _exact_store, "attend": _exact_attend, "found": _exact_found}[case["op"]](st)


def _codes(cache):
    return cache.float().double()


def _round_e4m3(x):
    """The nearest of the numbers with four significant bits from 2^-6 on and of the multiples of 2^-9 under it, ties to even."""
    step = torch.exp2((torch.frexp(x)[1] - 1).clamp(min=-6).double() - 3)
    return torch.round(x / step) * step


def _exact_store(st):
    """The rotation as a product of complex numbers, one block after the other."""
    n, rot, block = st["used"], 2 * st["cos"].shape[1], st["block"]
    unit = torch.complex(st["cos"].double(), st["sin"].double())[st["pos"][:n].long()][:, None, :]

    def turned(x, weight):
        x = x[:n].double()
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[-1] + EPS) * weight.double()
        lo, hi = (slice(0, rot, 2), slice(1, rot, 2)) if st["pairs"] else (slice(0, rot // 2), slice(rot // 2, rot))
        z = torch.complex(x[..., lo], x[..., hi]) * unit
        x[..., lo], x[..., hi] = z.real, z.imag
        return x

    q = torch.zeros(st["q"].shape, dtype=torch.float64, device=st["q"].device)
    q[:n] = turned(st["q"], st["q_weight"])
    page = st["k_cache"].shape[1]
    slots = st["slot"][:n].tolist()
    runs, begin = [], 0
    for i in range(1, n + 1):
        if i == n or slots[i] // block != slots[begin] // block:
            runs.append((begin, i))
            begin = i
    out = {"q": q}
    for name, x in (("k", turned(st["k"], st["k_weight"])), ("v", st["v"][:n].double())):
        codes, scale = _codes(st[name + "_cache"]), st[name + "_scale"].float().double()
        for a, b in runs:
            p, i = divmod(slots[a], page)
            c, f = divmod(i, block)
            largest = x[a:b].abs().amax((0, 2))
            s = torch.exp2((torch.frexp(largest)[1] - 1).double() - 7)
            if f:
                s = torch.maximum(s, scale[p, c])
                codes[p, i - f:i] = _round_e4m3(codes[p, i - f:i] * (scale[p, c] / s)[None, :, None])
            codes[p, i:i + b - a] = _round_e4m3(x[a:b] / s[None, :, None])
            scale[p, c] = s
        out[name + "_cache"], out[name + "_scale"] = codes, scale
    return out


def _exact_attend(st):
    """One request and key head at a time; masked keys are given no weight by a product with 0 and 1."""
    q, block = st["q"], st["block"]
    t, h, d = q.shape
    page, kv = st["k_cache"].shape[1:3]
    out = torch.zeros((t, h, d), dtype=torch.float64, device=q.device)
    lse = torch.zeros((t, h), dtype=torch.float64, device=q.device)
    begin = 0
    for r, (L, n) in enumerate(st["reqs"]):
        p = torch.arange(L, device=q.device)
        page_of, at = st["table"][r].long()[p // page], p % page
        ask = torch.arange(L - n, L, device=q.device)
        for c in range(kv):
            k, v = (_codes(st[x + "_cache"][:, :, c].view(torch.uint8)[page_of, at].view(CODE)) *
                    st[x + "_scale"].view(torch.uint8)[page_of, at // block, c].view(SCALE).float().double()[:, None] for x in "kv")
            for g in range(c * (h // kv), (c + 1) * (h // kv)):
                for a in range(0, n, 2048):
                    i = ask[a:a + 2048]
                    seen = (p[None, :] <= i[:, None]) & ((p[None, :] > i[:, None] - st["window"]) if st["window"] else True)
                    s = q[begin + a:begin + a + len(i), g].double() @ k.T * st["scale"]
                    top = torch.where(seen, s, torch.full_like(s, -1e300)).max(1).values
                    w = torch.exp(torch.minimum(s - top[:, None], torch.zeros_like(s))) * seen
                    z = w.sum(1)
                    out[begin + a:begin + a + len(i), g] = (w @ v) / z[:, None]
                    lse[begin + a:begin + a + len(i), g] = top + z.log()
        begin += n
    return {"out": out, "lse": lse}


def _exact_found(st):
    """The part before is one more key, with the score `lse` and the value `out`."""
    q, ids, block = st["q"], st["ids"].long(), st["block"]
    t, h, d = q.shape
    kv = st["keys"].shape[1]
    out = torch.zeros((t, h, d), dtype=torch.float64, device=q.device)
    lse = torch.zeros((t, h), dtype=torch.float64, device=q.device)
    for g in range(h):
        c = g // (h // kv)
        for a in range(0, t, 256):
            i = ids[a:a + 256, g]
            ok = i >= 0
            i = i.clamp(min=0)
            k, v = (_codes(st[x].view(torch.uint8)[i, c].view(CODE)) * st[y].view(torch.uint8)[i // block, c].view(SCALE).float().double()[..., None]
                    for x, y in (("keys", "k_scale"), ("values", "v_scale")))
            s = (k * q[a:a + 256, g, None].double()).sum(-1) * st["scale"]
            s = torch.cat([st["lse"][a:a + 256, g, None].double(), s], 1)
            ok = torch.cat([torch.ones_like(ok[:, :1]), ok], 1)
            v = torch.cat([st["out"][a:a + 256, g, None].double(), v], 1)
            z = torch.logsumexp(s.masked_fill(~ok, -math.inf), 1)
            w = torch.where(ok, torch.exp(s - z[:, None]), torch.zeros_like(s))
            out[a:a + 256, g] = (w[..., None] * v).sum(1)
            lse[a:a + 256, g] = z
    return {"out": out, "lse": lse}
