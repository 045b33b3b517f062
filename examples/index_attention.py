"""Decoding with a long past in an index.

    python examples/index_attention.py [--past 20000] [--steps 16]

A request's prompt goes through the paged cache in chunks.  Then its older part moves out: the keys of every key head become
the vectors of an index (inner products as distances, jx.mips_augment), the values stay in an array, and the pages go back to the
free ones.  Every further token attends to what is left in the cache and to the rows that a search with each query head finds,
joined.  What comes out is compared with attention over everything.

Projections and prompt are random; each past key is near some direction that queries take up again, as it is with the
keys that a model goes back to.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2601_07048_amd import jx  # noqa: E402

HEADS, KV_HEADS, DIM, PAGE = 8, 2, 64, 16


class Server:
    """One request: its paged cache, its table of pages and what has moved into an index."""

    def __init__(self, past, room, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.g, self.dtype = g, dtype
        pages = -(-(past + room) // PAGE) + 8
        self.k_cache, self.v_cache = (torch.zeros((pages, PAGE, KV_HEADS, DIM), dtype=dtype, device="cuda") for _ in range(2))
        self.table = torch.full((1, pages), -1, dtype=torch.int32, device="cuda")
        self.free = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        self.n_free = torch.tensor([pages], dtype=torch.int32, device="cuda")
        self.len = torch.zeros(1, dtype=torch.int32, device="cuda")
        angle = torch.arange(past + room, device="cuda", dtype=torch.float64)[:, None] * 1e6 ** (-torch.arange(0, DIM // 2, 2, device="cuda") / DIM)
        self.cos, self.sin = angle.cos().float(), angle.sin().float()  # half of each head turns
        self.weight = torch.ones(DIM, dtype=dtype, device="cuda")
        self.topics = torch.randn((256, DIM), generator=g, device="cuda")
        self.scale = 3.0 * DIM ** -0.5
        self.indices, self.moved = [], 0

    def project(self, tokens):
        """Stands for a layer's projections: queries, keys and values of new tokens."""
        def rows(heads, noise):
            topic = torch.randint(0, 256, (tokens, heads), generator=self.g, device="cuda")
            return (self.topics[topic] + noise * torch.randn((tokens, heads, DIM), generator=self.g, device="cuda")).to(self.dtype)

        return rows(HEADS, 0.3), rows(KV_HEADS, 0.6), torch.randn((tokens, KV_HEADS, DIM), generator=self.g, device="cuda").to(self.dtype)

    def step(self, tokens, k=64, L=128):
        """(out, log-sum-exp, queries, ids found) of `tokens` more tokens."""
        q, key, value = self.project(tokens)
        new = torch.full((1,), tokens, dtype=torch.int32, device="cuda")
        plan = jx.kv_plan(self.len, new, self.table, self.free, self.n_free, PAGE, tokens)
        # kv_len is 0 where there was no room: such a step leaves the request as it was (its results are zeros)
        self.n_free, self.len = plan.n_free, torch.where(plan.kv_len > 0, plan.kv_len, self.len)
        ready = jx.qk_norm_rope(q, key, value, self.k_cache, self.v_cache, plan.pos, plan.slot, self.cos, self.sin, self.weight, self.weight)
        part = jx.paged_attention(ready, self.k_cache, self.v_cache, self.table, plan.q_start, plan.kv_len, self.scale)
        if not self.moved:
            return (*part, ready, None)
        ids = torch.empty((tokens, HEADS, k), dtype=torch.int32, device="cuda")
        group = HEADS // KV_HEADS
        for c, index in enumerate(self.indices):
            asked = ready[:, c * group:(c + 1) * group].reshape(-1, DIM).float().contiguous()
            found, _ = index.search(jx.mips_augment(asked, is_query=True, dim_out=DIM + 4), k, L)
            ids[:, c * group:(c + 1) * group] = found.view(tokens, group, k)
        return (*jx.found_attention(ready, self.keys, self.values, ids, self.scale, part=part), ready, ids)

    def rows(self, first, end):
        """Keys and values of positions first .. end - 1, in order."""
        pages = self.table[0, first // PAGE:-(-end // PAGE)].long()
        return tuple(x[pages].flatten(0, 1)[first % PAGE:first % PAGE + end - first].clone() for x in (self.k_cache, self.v_cache))

    def move(self, tokens, R=32, L_build=64):
        """The first `tokens` (whole pages) leave the cache for an index for each key head."""
        assert tokens % PAGE == 0 and not self.moved
        self.keys, self.values = self.rows(0, tokens)
        for c in range(KV_HEADS):
            x = self.keys[:, c].float().contiguous()
            longest = float(jx.mips_augment(x, want_norms=True).max())
            index = jx.Index(DIM + 4, jx.F32, R, L_build, 1.2, capacity=tokens, max_batch=tokens)
            index.insert(jx.mips_augment(x, longest * 1.0001, dim_out=DIM + 4))
            self.indices.append(index)
        zero = torch.zeros(1, dtype=torch.int32, device="cuda")
        jx.kv_release(zero, zero + tokens // PAGE, self.table, self.free, self.n_free)
        self.moved = tokens


def over_all(server, ready):
    """Attention of the last token over everything, in 64 bits."""
    n = int(server.len)
    k, v = server.rows(server.moved, n)
    if server.moved:
        k, v = torch.cat([server.keys, k]), torch.cat([server.values, v])
    q = ready.double().view(-1, KV_HEADS, HEADS // KV_HEADS, DIM)
    s = torch.matmul(q[0], k.double().permute(1, 2, 0).contiguous()) * server.scale
    w = torch.softmax(s, -1)
    return torch.matmul(w, v.double().transpose(0, 1).contiguous()).reshape(1, HEADS, DIM), w.reshape(HEADS, n)


def main(past=20000, recent=400, steps=16, k=64, chunk=2048, quiet=False):
    past = past // PAGE * PAGE
    server = Server(past, recent + steps)
    done = 0
    while done < past + recent:
        tokens = min(chunk, past + recent - done)
        server.step(tokens)
        done += tokens
    server.move(past)
    worst, held = 0.0, []
    for _ in range(steps):
        out, lse, ready, ids = server.step(1, k=k)
        want, w = over_all(server, ready)
        worst = max(worst, float((out.double() - want).norm() / want.norm()))
        part = w[:, past:].sum(-1) + w[:, :past].gather(1, ids[0].long().clamp(min=0)).mul(ids[0] >= 0).sum(-1)
        held.append(float(part.mean()))
    if not quiet:
        print(f"{past} tokens in {KV_HEADS} indices, {recent} and more in {int((server.table >= 0).sum())} pages: "
              f"{k} rows found for each head and the cache hold {100 * sum(held) / len(held):.1f} % of the weights, "
              f"results within {100 * worst:.1f} % of attention over all")
    return worst, sum(held) / len(held)


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    ap.add_argument("--past", type=int, default=20000)
    ap.add_argument("--steps", type=int, default=16)
    ap.add_argument("--found", type=int, default=64)
    a = ap.parse_args()
    main(past=a.past, steps=a.steps, k=a.found)
