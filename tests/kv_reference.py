"""Plain 64-bit forms of the KV cache operators, request by request (numpy and
torch on the CPU), and the cases their tests share."""
import numpy as np
import torch

BLOCK = 16


def ref_tables(q_len, prev_len, table, free, n_tokens, group_start=None, prefix_len=None, prefix_blocks=None):
    """What kv_tables writes, in Python integers; table: list of rows, copied."""
    n = len(q_len)
    table = [list(r) for r in table]
    width = len(table[0]) if n else 0
    q_start, kv_len, positions, slots, taken = [0], [], [], [], 0
    for i in range(n):
        q, c = max(int(q_len[i]), 0), max(int(prev_len[i]), 0)
        pb = 0
        if group_start is not None and len(prefix_len):
            for g in range(len(prefix_len)):
                if group_start[g] <= i < group_start[g + 1]:
                    pb = min(max(int(prefix_len[g]), 0) // BLOCK, len(prefix_blocks[g]), width)
                    table[i][:pb] = prefix_blocks[g][:pb]
        first = min(max(-(-c // BLOCK), pb), width)
        for k in range(first, min(-(-(c + q) // BLOCK), width)):
            table[i][k] = free[taken] if taken < len(free) else -1
            taken += 1
        for t in range(q):
            p = c + t
            positions.append(p)
            b = table[i][p // BLOCK] if p // BLOCK < width else -1
            slots.append(b * BLOCK + p % BLOCK if b >= 0 else -1)
        kv_len.append(c + q)
        q_start.append(q_start[-1] + q)
    total = q_start[-1]
    positions = (positions + [-1] * n_tokens)[:n_tokens]
    slots = (slots + [-1] * n_tokens)[:n_tokens]
    return table, q_start, kv_len, positions, slots, [taken, total]


def ref_attend(q, k, v, table, q_start, kv_len, scale):
    """(out, lse) in 64 bits: q [rows, heads, d], k and v [block, kv head, 16, d] (CPU tensors)."""
    rows, heads, d = q.shape
    ratio = heads // k.shape[1]
    out = torch.zeros(rows, heads, d, dtype=torch.float64)
    lse = torch.full((rows, heads), -float("inf"), dtype=torch.float64)
    q = q.double()
    for i in range(len(kv_len)):
        length, new = int(kv_len[i]), int(q_start[i + 1] - q_start[i])
        if length <= 0 or new <= 0:
            continue
        blocks = torch.as_tensor([int(x) for x in table[i][:-(-length // BLOCK)]])
        keys = k[blocks].transpose(1, 2).reshape(-1, k.shape[1], d)[:length].double()
        values = v[blocks].transpose(1, 2).reshape(-1, k.shape[1], d)[:length].double()
        for h in range(heads):
            qs = q[int(q_start[i]):int(q_start[i + 1]), h]
            s = qs @ keys[:, h // ratio].T * scale
            past = torch.arange(length)[None] > (length - new + torch.arange(new))[:, None]
            s.masked_fill_(past, -float("inf"))
            row = ~past.all(1)
            at = int(q_start[i]) + torch.nonzero(row)[:, 0]
            lse[at, h] = torch.logsumexp(s[row], 1)
            out[at, h] = torch.softmax(s[row], 1) @ values[:, h // ratio]
    return out, lse


class Step:
    """Inputs of one attention step on the CPU, of the given lengths; block ids
    shuffled; everything outside the requests' tokens is NaN."""

    def __init__(self, seed, new, ctx, heads, kv_heads, dim, dtype, group_start=None, prefix=None, pad=0,
                 sharp=1.5, order="heads", offset=0, spare=3):
        r = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        n = len(new)
        self.kv_len = [c + q for c, q in zip(ctx, new)]
        self.q_start = [0]
        for q in new:
            self.q_start.append(self.q_start[-1] + q)
        self.rows = self.q_start[-1] + pad
        group_of = [-1] * n
        for gi in range(len(prefix or [])):
            for i in range(group_start[gi], group_start[gi + 1]):
                group_of[i] = gi
        width = max([1] + [-(-x // BLOCK) for x in self.kv_len] + [p // BLOCK for p in prefix or []])
        need = sum(-(-x // BLOCK) for x in self.kv_len) + sum(p // BLOCK for p in prefix or [])
        self.n_blocks = need + spare + offset
        ids = iter((r.permutation(need + spare) + offset).tolist())
        used = torch.zeros(self.n_blocks, dtype=torch.int64)
        self.prefix_blocks = [[next(ids) for _ in range(p // BLOCK)] for p in prefix or []]
        self.table = torch.full((n, width), -1, dtype=torch.int32)
        for i in range(n):
            row = list(self.prefix_blocks[group_of[i]]) if group_of[i] >= 0 else []
            # the prefix belongs to the row as a whole, also past the request's own length
            for k in range(-(-self.kv_len[i] // BLOCK)):
                if k >= len(row):
                    row.append(next(ids))
                used[row[k]] = max(int(used[row[k]]), min(BLOCK, self.kv_len[i] - k * BLOCK))
            self.table[i, :len(row)] = torch.tensor(row, dtype=torch.int32)
        for row in self.prefix_blocks:
            for b in row:
                used[b] = BLOCK
        self.group_start, self.prefix = group_start, prefix
        shape = (self.n_blocks, kv_heads, BLOCK, dim) if order == "heads" else (self.n_blocks, BLOCK, kv_heads, dim)
        self.k = torch.randn(shape, generator=g).to(dtype)
        self.v = torch.randn(shape, generator=g).to(dtype)
        if order == "tokens":
            self.k, self.v = self.k.transpose(1, 2), self.v.transpose(1, 2)
        empty = (torch.arange(BLOCK)[None] >= used[:, None])[:, None, :, None]
        self.k.masked_fill_(empty, float("nan"))
        self.v.masked_fill_(empty, float("nan"))
        self.q = (sharp * torch.randn(self.rows, heads, dim, generator=g)).to(dtype)
        self.scale = dim ** -0.5

    def expected(self):
        return ref_attend(self.q, self.k, self.v, self.table.tolist(), self.q_start, self.kv_len, self.scale)

    def to(self, rs, device="cuda"):
        """(cache, batch, q) on the device."""
        dev = lambda x: torch.tensor(x, dtype=torch.int32, device=device)  # noqa: E731
        k, v = self.k, self.v
        keep = lambda x: (x.to(device) if x.is_contiguous() else x.transpose(1, 2).contiguous().to(device).transpose(1, 2))  # noqa: E731
        cache = rs.KVCache(keep(k), keep(v))
        batch = rs.KVBatch(self.table.to(device), dev(self.q_start), dev(self.kv_len), self.rows,
                           dev(self.group_start) if self.prefix else None, dev(self.prefix) if self.prefix else None)
        return cache, batch, self.q.to(device)
