"""A worker's steps after the router: prompts are routed by the blocks that workers hold, and one worker then serves
its share from a paged KV cache: block tables and slot maps (kv_tables), the new tokens' K and V (kv_append), attention
that reads a shared template once for the requests on it (kv_attend); first the prompts, then single tokens.

    python examples/worker_steps.py

K, V and Q of a token are rows of fixed random matrices here (a stand-in for a layer's projections), so equal prefixes
have equal K and V, as in a model.  Every step's outputs are checked against plain attention in 64 bits.
"""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2606_17081_gb300 import routesim as rs  # noqa: E402
from paper_2606_17081_gb300 import workloads as wk  # noqa: E402

BLOCK, VOCAB = 16, 1000


def ints(x, dtype=torch.int32):
    return torch.tensor(x, dtype=dtype, device="cuda")


class Worker:
    """Host side of one worker: which block holds which block hash, which blocks are free, its requests."""

    def __init__(self, ctx, blocks=1024, heads=16, kv_heads=4, dim=64, dtype=torch.bfloat16):
        g = torch.Generator(device="cuda").manual_seed(1)
        self.ctx, self.heads, self.kv_heads, self.dim = ctx, heads, kv_heads, dim
        self.qkv = torch.randn(VOCAB, heads + 2 * kv_heads, dim, generator=g, device="cuda").to(dtype)
        store = torch.empty(blocks, 2, kv_heads, BLOCK, dim, dtype=dtype, device="cuda")
        self.cache = rs.KVCache(store[:, 0], store[:, 1])
        self.free = list(range(blocks))
        self.held = {}       # chained block hash -> block
        self.requests = []

    def admit(self, tokens, hashes):
        """A prompt; its leading blocks that are held already are shared."""
        known = 0
        while known < min(len(hashes), (len(tokens) - 1) // BLOCK) and hashes[known] in self.held:
            known += 1
        self.requests.append({"tokens": list(tokens), "hashes": list(hashes), "cached": known * BLOCK,
                              "blocks": [self.held[h] for h in hashes[:known]]})

    def step(self):
        """All tokens that are not cached yet, of every request.  Returns (out, lse) and the rows' starts."""
        # requests on one template beside each other; they share the blocks that all of them have cached
        self.requests.sort(key=lambda r: r["blocks"][:1])
        starts, prefixes = [0], []
        for i, r in enumerate(self.requests):
            first = self.requests[starts[-1]]
            if i > starts[-1] and r["blocks"][:1] != first["blocks"][:1]:
                starts.append(i)
        starts.append(len(self.requests))
        for a, b in zip(starts, starts[1:]):
            rows = [r["blocks"][:r["cached"] // BLOCK] for r in self.requests[a:b]]
            n = 0
            while b - a > 1 and all(len(x) > n and x[n] == rows[0][n] for x in rows):
                n += 1
            prefixes.append(rows[0][:n])
        new = [len(r["tokens"]) - r["cached"] for r in self.requests]
        width = max(-(-len(r["tokens"]) // BLOCK) for r in self.requests)
        longest = max(max(map(len, prefixes)), 1)
        table = ints([r["blocks"] + [-1] * (width - len(r["blocks"])) for r in self.requests])
        n, rows = len(new), sum(new)
        batch = rs.KVBatch(table, ints([0] * (n + 1)), ints([0] * n), rows, ints(starts), ints([len(p) * BLOCK for p in prefixes]))
        positions, slots, counts = ints([0] * rows), ints([0] * rows, torch.int64), ints([0, 0], torch.int64)
        rs.kv_tables(self.ctx.h, batch, ints(new), ints([r["cached"] for r in self.requests]),
                     ints([p + [-1] * (longest - len(p)) for p in prefixes]), ints(self.free), positions, slots, counts)
        tokens = ints([t for r in self.requests for t in r["tokens"][r["cached"]:]], torch.int64)
        qkv = self.qkv[tokens]
        h, k = self.heads, self.kv_heads
        rs.kv_append(self.ctx.h, self.cache, qkv[:, h:h + k], qkv[:, h + k:], slots)
        out = torch.empty(rows, h, self.dim, dtype=qkv.dtype, device="cuda")
        lse = torch.empty(rows, h, device="cuda")
        rs.kv_attend(self.ctx.h, self.cache, batch, qkv[:, :h], self.dim ** -0.5, out, lse)
        # what the host keeps: the blocks, and the full ones under their hashes
        taken = int(counts[0])
        assert taken <= len(self.free), "the cache is full"
        self.free = self.free[taken:]
        for r, row in zip(self.requests, table.tolist()):
            r["blocks"] = row[:-(-len(r["tokens"]) // BLOCK)]
            r["cached"] = len(r["tokens"])
            for x, b in zip(r["hashes"], r["blocks"]):
                self.held.setdefault(x, b)
        return out, lse, np.cumsum([0] + new), [len(p) for p in prefixes]

    def expected(self, r, rows):
        """Plain attention of a request's last `rows` tokens, in 64 bits."""
        x = self.qkv[ints(r["tokens"], torch.int64)].double()
        h, k, n = self.heads, self.kv_heads, len(r["tokens"])
        q, keys, values = x[n - rows:, :h], x[:, h:h + k], x[:, h + k:]
        keys, values = (y.repeat_interleave(h // k, 1) for y in (keys, values))
        s = torch.einsum("qhd,khd->hqk", q, keys) * self.dim ** -0.5
        s.masked_fill_(torch.arange(n, device="cuda")[None] > torch.arange(n - rows, n, device="cuda")[:, None], -float("inf"))
        return torch.einsum("hqk,khd->qhd", torch.softmax(s, -1), values)


def main(n_prompts=24, steps=4, W=2) -> float:
    spec = wk.TraceSpec(n_req=n_prompts, len_kind="uniform", len_min=300, len_max=700, n_groups=3, prefix_min=200,
                        prefix_max=280, vocab=VOCAB, out_kind="uniform", out_min=1, out_max=9)
    trace = wk.make_trace(spec, 5)
    dev = rs.device_trace(trace)
    ctx = rs.Context(W=W, K=1024, n_instances=1)
    n = trace.n_req
    hashes = torch.zeros(trace.n_tokens // BLOCK + 1, dtype=torch.int64, device="cuda")
    rs.route_hash_blocks(ctx.h, dev.tokens, dev.offsets, n, hashes)
    chosen, prefix = ints([0] * n), ints([0] * n * W)
    rs.route_batch(ctx.h, 0, dev.tokens, dev.offsets, n, dev.out_len, chosen, None, prefix)
    rs.route_active(ctx.h, 0, W)   # (reports what the routing found wrong)
    chosen, prefix = chosen.cpu().numpy(), prefix.cpu().numpy().reshape(n, W)
    hashes = hashes.cpu().numpy()
    mine = [i for i in range(n) if chosen[i] == chosen[0]]
    print(f"{len(mine)} of {n} prompts go to worker {chosen[0]}; the router found {prefix[mine, chosen[0]].tolist()} blocks cached")

    worker = Worker(ctx)
    worst = 0.0

    def check(what):
        nonlocal worst
        out, _, start, shared = worker.step()
        err = 0.0
        for i, r in enumerate(worker.requests):
            if start[i] == start[i + 1]:
                continue   # (nothing new in this step)
            want = worker.expected(r, start[i + 1] - start[i])
            err = max(err, float((out[start[i]:start[i + 1]].double() - want).abs().max()))
        worst = max(worst, err)
        print(f"{what}: {start[-1]} tokens, shared blocks of the groups {shared}, largest difference {err:.1e}")

    def prompt(i):
        a, b = trace.offsets[i], trace.offsets[i + 1]
        worker.admit(trace.tokens[a:b].tolist(), hashes[a // BLOCK:a // BLOCK + (b - a) // BLOCK].tolist())

    # the first prompt on each template, then the others, which find the template's blocks held
    first = {trace.group[i]: i for i in reversed(mine)}
    for i in first.values():
        prompt(i)
    check("first prompts")
    for i in mine:
        if i not in first.values():
            prompt(i)
    check("their followers")
    draw = np.random.default_rng(3)
    for k in range(steps):
        for r in worker.requests:
            r["tokens"].append(int(draw.integers(VOCAB)))
        check(f"single tokens {k + 1}")
    ctx.close()
    return worst


if __name__ == "__main__":
    main()
