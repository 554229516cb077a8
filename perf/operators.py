"""Measured operators of a worker's paged KV cache: what follows when a router has sent requests to the worker.

Kinds of case ("kind"):

  tables  kv_tables: block tables, positions and slot maps of one step, from the requests' lengths
  append  kv_append: the step's new K and V into the cache's blocks, through the slot map
  attend  kv_attend: causal attention of the step's tokens over the blocks; requests of a group share a prefix

A case's lengths follow from the case alone ("lens" seeds them), so that its work is known; where the blocks lie and
what the tensors hold follow from the seed.  A request's context is its group's prefix and then its own tokens, "own_lo"
to "own_hi" of them (evenly spread over the logarithm), and it brings "q_lo" to "q_hi" new tokens.  "pad" rows at the end of
the token dimension belong to no request, as in a step of fixed size.  What no request has written in the cache is NaN:
memory that the cache has not used yet can hold anything.
"""
import math
import random

import torch

own = False

DEV = "cuda"
BLOCK = 16
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
_context = None   # the worker's context of the library, one for the process


def _attend(name, n, heads, kv_heads, dim, dtype, **more):
    c = {"name": name, "kind": "attend", "n": n, "heads": heads, "kv_heads": kv_heads, "dim": dim, "dtype": dtype,
         "groups": 1, "prefix": 0, "own_lo": 1, "own_hi": 1, "q_lo": 1, "q_hi": 1, "pad": 0, "order": "heads", "lens": 1}
    c.update(more)
    return c


def _tables(name, n, **more):
    c = {"name": name, "kind": "tables", "n": n, "groups": 1, "prefix": 0, "own_lo": 1, "own_hi": 1, "q_lo": 1, "q_hi": 1,
         "pad": 0, "lens": 1}
    c.update(more)
    return c


def _append(name, n, kv_heads, dim, dtype, **more):
    c = {"name": name, "kind": "append", "n": n, "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "pad": 0, "order": "heads"}
    c.update(more)
    return c


def listed():
    return [
        # the step of a batch of single tokens: launches and latency
        _tables("tables_tokens", 64, groups=4, prefix=2048, own_lo=1, own_hi=2048, pad=3),
        # a large step of whole prompts on 64 templates
        _tables("tables_prompts", 1024, groups=64, prefix=2048, own_lo=16, own_hi=2048, q_lo=1, q_hi=511),
        # the new tokens of a decoding batch
        _append("append_tokens", 64, 8, 128, "bf16"),
        # the new tokens of a step of prompts, token-major blocks
        _append("append_prompts", 16001, 8, 128, "bf16", pad=31, order="tokens"),
        # one conversation, one token: the smallest call
        _attend("one_token", 1, 32, 8, 128, "bf16", groups=0, own_lo=700, own_hi=700),
        # a few requests on one template
        _attend("few_shared", 8, 32, 8, 128, "bf16", prefix=1024, own_lo=16, own_hi=512),
        # a decoding batch on one long document: the prefix's products are the work
        _attend("long_shared", 64, 64, 8, 128, "bf16", prefix=32768, own_lo=16, own_hi=1024),
        # a large decoding batch on eight templates: the requests' own blocks are the work
        _attend("many_groups", 256, 32, 8, 128, "bf16", groups=8, prefix=2048, own_lo=256, own_hi=8192, order="tokens", pad=13),
        # a few proposed tokens a request, one kv head for each head, small heads, 16-bit floats
        _attend("proposed_fp16", 48, 16, 16, 64, "fp16", groups=2, prefix=4096, own_lo=1, own_hi=900, q_lo=1, q_hi=5),
        # seven heads a kv head
        _attend("odd_heads", 33, 28, 4, 128, "bf16", groups=3, prefix=4992, own_lo=1, own_hi=300, pad=2),
        # prompts that find a template cached and bring the rest
        _attend("prompts_shared", 6, 32, 8, 128, "bf16", prefix=2048, own_lo=0, own_hi=0, q_lo=100, q_hi=2047),
        # one piece of a long prompt: bound by products
        _attend("prompt_piece", 1, 32, 8, 128, "bf16", groups=0, own_lo=12288, own_hi=12288, q_lo=4096, q_hi=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        most[c["kind"]] = {k: max(most.get(c["kind"], {}).get(k, 0), w[k]) for k in w}
    while True:
        c = _drawn(rng)
        w = work(c)
        if all(w[k] <= most[c["kind"]][k] for k in w):
            return c


def _drawn(rng):
    kind = rng.choice(["tables", "append", "attend", "attend", "attend", "attend"])
    pad = rng.choice([0, 0, rng.randint(1, 40)])
    lens = rng.randrange(1 << 20)
    if kind == "tables":
        c = _tables("", _log(rng, 1, 1500), groups=rng.choice([0, 1, rng.randint(2, 64)]), prefix=16 * _log(rng, 1, 128), own_lo=1, own_hi=_log(rng, 1, 8192),
                    q_lo=rng.choice([0, 1]), q_hi=rng.choice([1, _log(rng, 1, 600)]), pad=pad, lens=lens)
    elif kind == "append":
        c = _append("", _log(rng, 1, 16000), rng.choice([1, 2, 4, 5, 8, 16]), rng.choice([64, 128]), rng.choice(["bf16", "fp16"]), pad=pad,
                    order=rng.choice(["heads", "tokens"]))
    else:
        kv_heads = rng.choice([1, 2, 4, 8, 8, 16])
        ratio = rng.choice([1, 2, 3, 4, 5, 7, 8])
        more = {"order": rng.choice(["heads", "tokens"]), "pad": pad, "lens": lens}
        form = rng.choice(["shared", "groups", "alone", "few", "prompts"])
        n = _log(rng, 1, 256)
        if form == "prompts":
            n = rng.randint(1, 6)
            more.update(groups=rng.choice([0, 1]), prefix=16 * _log(rng, 1, 256), own_lo=0, own_hi=_log(rng, 1, 2048), q_lo=_log(rng, 1, 100), q_hi=_log(rng, 100, 2100))
        elif form == "alone":
            more.update(groups=0, own_lo=1, own_hi=_log(rng, 1, 8192))
        else:
            groups = 1 if form == "shared" else rng.randint(1, min(n, 12))
            more.update(groups=groups, prefix=16 * _log(rng, 1, 2048 if form == "shared" else 256), own_lo=1, own_hi=_log(rng, 1, 2048))
            if form == "few":
                more.update(q_lo=rng.choice([0, 1]), q_hi=rng.randint(2, 8))
        c = _attend("", n, kv_heads * ratio, kv_heads, rng.choice([64, 128, 128]), rng.choice(["bf16", "bf16", "fp16"]), **more)
    del c["name"]
    return c


# ------------------------------------------------------------------ a case's lengths

def _lengths(case):
    """Of every request: new tokens, context before them, group; of every group: first request, shared prefix (in tokens, whole blocks)."""
    r = random.Random(case["lens"])
    n, groups = case["n"], min(case["groups"], case["n"])
    cuts = sorted(r.sample(range(1, n), groups - 1)) if groups > 1 else []
    start = [0] + cuts + [n] if groups else []
    prefix = [case["prefix"] if g == 0 else (r.randint(case["prefix"] // 2, case["prefix"]) // BLOCK) * BLOCK for g in range(groups)]
    group = [g for g in range(groups) for _ in range(start[g], start[g + 1])] or [-1] * n
    lo, hi = case["own_lo"], max(case["own_lo"], case["own_hi"])
    ctx = [(prefix[g] if g >= 0 else 0) + (min(hi, _log(r, lo + 1, hi + 1) - 1) if hi else 0) for g in group]
    new = [r.randint(case["q_lo"], max(case["q_lo"], case["q_hi"])) for _ in range(n)]
    new[0] += not any(new)
    return new, ctx, group, start, prefix


def _blocks(tokens):
    return -(-tokens // BLOCK)


def work(case):
    if case["kind"] == "append":
        row = case["kv_heads"] * case["dim"] * 2 * 2
        return {"bytes": case["n"] * (2 * row + 8) + 8 * case["pad"], "flops": 0}
    new, ctx, group, start, prefix = _lengths(case)
    pre = [prefix[g] if g >= 0 else 0 for g in group]
    if case["kind"] == "tables":
        fresh = sum(max(0, _blocks(c + q) - max(_blocks(c), p // BLOCK)) for q, c, p in zip(new, ctx, pre))
        kept = sum(1 for q, c, p in zip(new, ctx, pre) if q and c % BLOCK and c >= p)
        rows = sum(new) + case["pad"]
        # lengths, prefix lists and free blocks read; table entries, starts and lengths, positions and slots written
        return {"bytes": 8 * len(new) + 4 * sum(prefix) // BLOCK + 8 * len(start) + 8 * fresh + 4 * kept + 4 * sum(pre) // BLOCK + 8 * len(new) + 12 * rows + 16, "flops": 0}
    used = [g for g in range(len(prefix)) if sum(new[start[g]:start[g + 1]])]
    keys = sum(prefix[g] for g in used) + sum(c + q - p for q, c, p in zip(new, ctx, pre) if q)
    pairs = sum(q * c + q * (q + 1) // 2 for q, c in zip(new, ctx))
    rows = sum(new) + case["pad"]
    entries = sum(_blocks(c + q) - p // BLOCK for q, c, p in zip(new, ctx, pre) if q) + sum(prefix[g] // BLOCK for g in used)
    # K and V of every distinct token, q, the output and its log sums, table entries and lengths
    return {"bytes": keys * case["kv_heads"] * case["dim"] * 4 + rows * case["heads"] * (case["dim"] * 4 + 4) + 4 * entries + 12 * len(new),
            "flops": 4 * case["dim"] * case["heads"] * pairs}


# ------------------------------------------------------------------ inputs

def _ints(v, kind=torch.int32):
    return torch.tensor(v, dtype=kind, device=DEV)


def _cache(case, n_blocks):
    """An empty cache of either order, as [block, head, token in block, element]; K and V of a block beside each other."""
    h, d, t = case["kv_heads"], case["dim"], TYPES[case["dtype"]]
    if case["order"] == "heads":
        both = torch.empty(n_blocks, 2, h, BLOCK, d, dtype=t, device=DEV)
        return both[:, 0], both[:, 1], both
    both = torch.empty(n_blocks, 2, BLOCK, h, d, dtype=t, device=DEV)
    return both[:, 0].transpose(1, 2), both[:, 1].transpose(1, 2), both


def prepare(case, seed):
    r = torch.Generator(device=DEV).manual_seed(int(seed))
    s = {"kind": case["kind"]}
    if case["kind"] == "append":
        n, h, d = case["n"], case["kv_heads"], case["dim"]
        n_blocks = _blocks(n) + _blocks(n) // 4 + 1
        s["k"], s["v"], both = _cache(case, n_blocks)
        both.zero_()
        # k and v as a projection leaves them: columns of one matrix, after four heads of q for each of theirs
        qkv = torch.randn(n + case["pad"], 6 * h, d, generator=r, device=DEV).to(TYPES[case["dtype"]])
        s["k_new"], s["v_new"] = qkv[:, 4 * h:5 * h], qkv[:, 5 * h:]
        slots = torch.randperm(n_blocks, generator=r, device=DEV)[:_blocks(n), None] * BLOCK + torch.arange(BLOCK, device=DEV)
        s["slots"] = torch.cat([slots.reshape(-1)[:n], _ints([-1] * case["pad"], torch.int64)])
        return _with_handles(s)
    new, ctx, group, start, prefix = _lengths(case)
    n, rows = len(new), sum(new) + case["pad"]
    pre = [prefix[g] if g >= 0 else 0 for g in group]
    whole = case["kind"] == "attend"   # the tables of the step's end, or those of its start
    ends = [max(_blocks(c + q) if whole else _blocks(c), p // BLOCK) for q, c, p in zip(new, ctx, pre)]
    owned = _ints([e - p // BLOCK for e, p in zip(ends, pre)], torch.int64)
    fresh = 0 if whole else sum(max(0, _blocks(c + q) - e) for q, c, e in zip(new, ctx, ends))
    shared, taken = sum(prefix) // BLOCK, int(sum(ends)) - sum(pre) // BLOCK
    n_blocks = shared + taken + fresh + 7 + n // 4
    ids = torch.randperm(n_blocks, generator=r, device=DEV).to(torch.int32)
    width = max(max(_blocks(c + q) for q, c in zip(new, ctx)), max(pre) // BLOCK, 1)
    # the prefixes' blocks, the requests' own, and then the free ones, in the order of ids
    lists = torch.full((max(len(prefix), 1), max(max(prefix, default=0) // BLOCK, 1)), -1, dtype=torch.int32, device=DEV)
    col = torch.arange(max(width, lists.shape[1]), device=DEV)
    if prefix:
        per = _ints([p // BLOCK for p in prefix], torch.int64)
        at = (torch.cumsum(per, 0) - per)[:, None] + col[None, :lists.shape[1]]
        lists = torch.where(col[None, :lists.shape[1]] < per[:, None], ids[at.clamp(max=n_blocks - 1)], lists)
    p_blocks = _ints([p // BLOCK for p in pre], torch.int64)[:, None]
    own_at = shared + (torch.cumsum(owned, 0) - owned)[:, None] + col[None, :width] - p_blocks
    mine = (col[None, :width] >= p_blocks) & (col[None, :width] < p_blocks + owned[:, None])
    table = torch.where(mine, ids[own_at.clamp(0, n_blocks - 1)], _ints(-1))
    if whole and prefix:
        got = lists[_ints(group, torch.int64)][:, :width]
        got = torch.nn.functional.pad(got, (0, width - got.shape[1]))
        table = torch.where(col[None, :width] < p_blocks, got, table)
    s.update(table=table.contiguous(), group_start=_ints(start) if start else None, prefix_len=_ints(prefix) if start else None, rows=rows)
    if not whole:
        s.update(q_len=_ints(new), prev_len=_ints(ctx), prefix_blocks=lists.contiguous() if start else None, free=ids[shared + taken:].contiguous(),
                 q_start=torch.zeros(n + 1, dtype=torch.int32, device=DEV), kv_len=torch.zeros(n, dtype=torch.int32, device=DEV))
        return _with_handles(s)
    s["q_start"] = torch.nn.functional.pad(torch.cumsum(_ints(new), 0), (1, 0)).to(torch.int32)
    s["kv_len"] = _ints([q + c for q, c in zip(new, ctx)])
    k, v, both = _cache(case, n_blocks)
    both.normal_(generator=r)
    # nothing has been written outside the prefixes' blocks and the requests' own tokens
    used = torch.zeros(n_blocks, dtype=torch.int64, device=DEV)
    used[ids[:shared].long()] = BLOCK
    fill = (s["kv_len"][:, None] - col[None, :width] * BLOCK).clamp(0, BLOCK)
    used[table[mine].long()] = fill[mine].long()
    empty = torch.arange(BLOCK, device=DEV)[None] >= used[:, None]
    k.masked_fill_(empty[:, None, :, None], math.nan)
    v.masked_fill_(empty[:, None, :, None], math.nan)
    h, d = case["heads"], case["dim"]
    # heads that look far around them and heads that look at little: scores of a deviation of 0.5 to 3
    sharp = torch.empty(1, h, 1, device=DEV).uniform_(0.5, 3.0, generator=r)
    qkv = torch.randn(rows, h + 2 * case["kv_heads"], d, generator=r, device=DEV)
    qkv[:, :h] *= sharp
    s.update(k=k, v=v, q=qkv.to(TYPES[case["dtype"]])[:, :h], scale=1.0 / math.sqrt(d))
    # what the step's scheduler knows on the host: the longest of each
    sizes = [sum(new[a:b]) for a, b in zip(start, start[1:])]
    s.update(max_q=max(new), max_own=max(c + q - p for q, c, p in zip(new, ctx, pre)), max_prefix=max(prefix, default=0), max_group=max(sizes, default=0))
    return _with_handles(s)


def _with_handles(s):
    """The library's descriptors of the program's buffers (pointers and strides, no values), which it keeps with them."""
    global _context
    if own:
        from paper_2606_17081_gb300 import routesim as rs
        if _context is None:
            _context = rs.Context(W=1, K=65536, stream=torch.cuda.current_stream().cuda_stream)
        if "k" in s:
            s["cache"] = rs.KVCache(s["k"], s["v"])
        if "table" in s:
            s["batch"] = rs.KVBatch(s["table"], s["q_start"], s["kv_len"], s["rows"], s["group_start"], s["prefix_len"])
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    if not own:
        return {"tables": _plain_tables, "append": _plain_append, "attend": _plain_attend}[s["kind"]](s)
    from paper_2606_17081_gb300 import routesim as rs
    if s["kind"] == "append":
        rs.kv_append(_context.h, s["cache"], s["k_new"], s["v_new"], s["slots"])
        return {"k": s["k"], "v": s["v"]}
    if s["kind"] == "attend":
        out = torch.empty(s["q"].shape, dtype=s["q"].dtype, device=DEV)
        lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=DEV)
        rs.kv_attend(_context.h, s["cache"], s["batch"], s["q"], s["scale"], out, lse)
        return {"out": out, "lse": lse}
    positions = torch.empty(s["rows"], dtype=torch.int32, device=DEV)
    slots = torch.empty(s["rows"], dtype=torch.int64, device=DEV)
    counts = torch.empty(2, dtype=torch.int64, device=DEV)
    rs.kv_tables(_context.h, s["batch"], s["q_len"], s["prev_len"], s["prefix_blocks"], s["free"], positions, slots, counts)
    return {"table": s["table"], "q_start": s["q_start"], "kv_len": s["kv_len"], "positions": positions, "slots": slots, "counts": counts}


def _groups_of(s, n):
    """Of every request its group and the group's prefix in tokens; no groups: 0 and 0."""
    if s["group_start"] is None:
        return torch.zeros(n, dtype=torch.int64, device=DEV), torch.zeros(n, dtype=torch.int64, device=DEV)
    group = torch.searchsorted(s["group_start"][1:].contiguous(), torch.arange(n, dtype=torch.int32, device=DEV), right=True)
    return group, s["prefix_len"].long()[group] // BLOCK * BLOCK


def _rows_of(q_start, rows):
    """Of every row its request, its token there, and whether it has a request."""
    row = torch.arange(rows, device=DEV, dtype=torch.int32)
    req = torch.searchsorted(q_start[1:].contiguous(), row, right=True).clamp(max=q_start.numel() - 2)
    return req, row - q_start[req], row < q_start[-1]


def _plain_tables(s):
    table, n = s["table"], s["q_len"].numel()
    q, c = s["q_len"].long(), s["prev_len"].long()
    s["q_start"][1:] = torch.cumsum(q, 0)
    s["kv_len"].copy_(c + q)
    group, pre = _groups_of(s, n)
    col = torch.arange(table.shape[1], device=DEV)[None]
    if s["prefix_blocks"] is not None:
        lists = torch.nn.functional.pad(s["prefix_blocks"], (0, max(0, table.shape[1] - s["prefix_blocks"].shape[1])))[:, :table.shape[1]]
        table.copy_(torch.where(col < (pre // BLOCK)[:, None], lists[group], table))
    first = torch.maximum((c + BLOCK - 1) // BLOCK, pre // BLOCK)
    count = ((c + q + BLOCK - 1) // BLOCK - first).clamp(min=0)
    at = (torch.cumsum(count, 0) - count)[:, None] + col - first[:, None]
    fresh = (col >= first[:, None]) & (col < (first + count)[:, None])
    got = torch.where(at < s["free"].numel(), s["free"][at.clamp(0, s["free"].numel() - 1)], -1)
    table.copy_(torch.where(fresh, got, table))
    req, t, valid = _rows_of(s["q_start"], s["rows"])
    pos = torch.where(valid, c[req] + t, 0)
    block = table[req, pos // BLOCK].long()
    slots = torch.where(valid & (block >= 0), block * BLOCK + pos % BLOCK, -1)
    return {"table": table, "q_start": s["q_start"], "kv_len": s["kv_len"], "positions": torch.where(valid, pos, -1).to(torch.int32), "slots": slots,
            "counts": torch.stack([count.sum(), q.sum()])}


def _plain_append(s):
    # a row without a slot writes the same as the row of the highest slot
    last = s["slots"].argmax()
    row = torch.where(s["slots"] >= 0, torch.arange(s["slots"].numel(), device=DEV), last)
    slot = s["slots"][row]
    s["k"][slot // BLOCK, :, slot % BLOCK] = s["k_new"][row]
    s["v"][slot // BLOCK, :, slot % BLOCK] = s["v_new"][row]
    return {"k": s["k"], "v": s["v"]}


def _spread(x, a, b, shape):
    """zeros(shape + ...) with x[i] at [a[i], b[i]]; a[i] = shape[0]: nowhere."""
    out = torch.zeros(shape[0] + 1, shape[1], *x.shape[1:], dtype=x.dtype, device=DEV)
    out[a, b] = x
    return out[:-1]


def _shared_keys(s, q, limit, a, b, shape, blocks, keys):
    """(m, l, o) of every row over lists of blocks [shape[0], count] that hold keys [shape[0]] tokens: row i takes list a[i], b[i]-th of its rows."""
    hk, ratio, d = q.shape[1:]
    queries = _spread(q, a, b, shape).transpose(1, 2).flatten(2, 3)
    limits = _spread(limit, a, b, shape).repeat_interleave(ratio, 1)[:, None, :, None]
    part = _part(queries, _keys(s["k"], blocks, keys), _keys(s["v"], blocks, keys), limits, s["scale"])
    return [x.reshape(shape[0], hk, shape[1], ratio, -1)[a.clamp(max=shape[0] - 1), :, b] for x in part]


def _part(q, k, v, limit, scale):
    """(m, l, o) of one part of the keys: q [b, h, rows, d], k and v [b, h, keys, d], row r sees keys below limit [b, 1, rows, 1]."""
    score = torch.matmul(q, k.transpose(-1, -2)) * scale
    seen = torch.arange(k.shape[2], device=DEV) < limit
    score = torch.where(seen, score, -math.inf)
    m = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(m == -math.inf, 0.0, m))
    return m, p.sum(-1, keepdim=True), torch.matmul(p, v)


def _keys(cache, blocks, keys):
    """[b, h, tokens, d] of lists of blocks [b, count] in 32 bits; 0 where a list has fewer tokens than keys [b]."""
    x = cache[blocks.clamp(min=0)].float().transpose(1, 2).flatten(2, 3)
    return torch.where(torch.arange(x.shape[2], device=DEV)[None, None, :, None] < keys[:, None, None, None], x, 0.0)


def _plain_attend(s):
    q, n, hk = s["q"], s["kv_len"].numel(), s["k"].shape[1]
    rows, heads, d = q.shape
    ratio = heads // hk
    req, t, valid = _rows_of(s["q_start"], rows)
    kv_len, new = s["kv_len"].long(), (s["q_start"][1:] - s["q_start"][:-1]).long()
    limit = torch.where(valid, (kv_len - new)[req] + t + 1, 0)
    group, pre = _groups_of(s, n)
    qf = q.float().reshape(rows, hk, ratio, d)
    # the requests' own keys, padded to the longest list and the most tokens
    at = (pre // BLOCK)[:, None] + torch.arange(_blocks(s["max_own"]), device=DEV)
    blocks = torch.gather(s["table"], 1, at.clamp(max=s["table"].shape[1] - 1)).long()
    parts = [_shared_keys(s, qf, limit - pre[req], torch.where(valid, req, n), torch.where(valid, t, 0), (n, max(s["max_q"], 1)), blocks, kv_len - pre)]
    if s["max_prefix"]:
        # the groups' prefixes, each once for all its rows
        first = s["group_start"][:-1].long()
        keys = s["prefix_len"].long() // BLOCK * BLOCK
        in_group = torch.arange(rows, device=DEV) - s["q_start"].long()[first][group[req]]
        parts.append(_shared_keys(s, qf, torch.minimum(limit, keys[group[req]]), torch.where(valid, group[req], first.numel()), torch.where(valid, in_group, 0),
                                  (first.numel(), max(s["max_group"], 1)), s["table"][first][:, :_blocks(s["max_prefix"])].long(), keys))
    m = torch.stack([p[0] for p in parts]).amax(0)
    w = [torch.where(p[0] == -math.inf, 0.0, torch.exp(p[0] - m)) for p in parts]
    l = sum(x * p[1] for x, p in zip(w, parts))
    o = sum(x * p[2] for x, p in zip(w, parts))
    some = valid[:, None, None, None] & (l > 0)
    out = torch.where(some, o / torch.where(some, l, 1.0), 0.0)
    lse = torch.where(some, m + torch.log(torch.where(some, l, 1.0)), -math.inf)
    return {"out": out.reshape(rows, heads, d).to(q.dtype), "lse": lse.reshape(rows, heads)}


# ------------------------------------------------------------------ 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "tables":
        return None   # whole numbers
    if case["kind"] == "append":
        k, v = s["k"].double(), s["v"].double()
        rows = [r for r in range(s["slots"].numel()) if r < case["n"]]
        slot = s["slots"][rows]
        for h in range(case["kv_heads"]):
            k[slot // BLOCK, h, slot % BLOCK] = s["k_new"][rows, h].double()
            v[slot // BLOCK, h, slot % BLOCK] = s["v_new"][rows, h].double()
        return {"k": k, "v": v}
    rows, heads, d = s["q"].shape
    ratio = heads // case["kv_heads"]
    out = torch.zeros(rows, heads, d, dtype=torch.float64, device=DEV)
    lse = torch.full((rows, heads), -math.inf, dtype=torch.float64, device=DEV)
    at = 0
    for i, (length, new) in enumerate(zip(s["kv_len"].tolist(), (s["q_start"][1:] - s["q_start"][:-1]).tolist())):
        blocks = s["table"][i, :_blocks(length)].long()
        keys = s["k"][blocks].transpose(1, 2).reshape(-1, case["kv_heads"], d)[:length].double()
        values = s["v"][blocks].transpose(1, 2).reshape(-1, case["kv_heads"], d)[:length].double()
        for a in range(0, new, 512):
            b = min(new, a + 512)
            seen = length - new + b
            past = torch.arange(seen, device=DEV)[None] > length - new + torch.arange(a, b, device=DEV)[:, None]
            for h in range(heads):
                score = s["q"][at + a:at + b, h].double() @ keys[:seen, h // ratio].T * s["scale"]
                score.masked_fill_(past, -math.inf)
                lse[at + a:at + b, h] = torch.logsumexp(score, 1)
                out[at + a:at + b, h] = torch.softmax(score, 1) @ values[:seen, h // ratio]
        at += new
    return {"out": out, "lse": lse}
