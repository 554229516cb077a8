"""Steps whose rows end inside a request: kv_tables leaves the tokens past the last row out, and kv_append and kv_attend
follow it.  Values against the definition in 64 bits, bounds as in test_gpu_kv_attend; the cache holds NaN wherever the
step or the cached tokens have written nothing."""
import random

import pytest

from kv_reference import BLOCK, ref_attend
from paper_2606_17081_gb300 import routesim as rs

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

from test_gpu_kv_attend import BF, compare, ctx  # noqa: E402, F401


class Chain:
    """What compare asks of a step."""

    def expected(self):
        return ref_attend(self.q, self.k, self.v, self.table.tolist(), self.q_start, self.kv_len, self.scale)


def cut_step(ctx, seed, new, past, rows, heads, kv_heads, dim, dtype, prefix=0):  # noqa: F811
    """The first `rows` rows of a step through the three operators; the request in which they end, and later ones, keep
    the positions of the whole step.  prefix: cached tokens that all requests share."""
    n = len(new)
    dev = lambda x, t=torch.int32: torch.tensor(x, dtype=t, device="cuda")  # noqa: E731
    g = torch.Generator().manual_seed(seed)
    width = max(-(-(a + b) // BLOCK) for a, b in zip(new, past))
    blocks = prefix // BLOCK + n * width + 2
    ids = random.Random(seed).sample(range(blocks), blocks)
    shared, rest = ids[:prefix // BLOCK], ids[prefix // BLOCK:]
    k, v = (torch.full((blocks, kv_heads, BLOCK, dim), float("nan")) for _ in range(2))
    table = []
    for i in range(n):
        row = list(shared)
        while len(row) * BLOCK < past[i]:
            row.append(rest.pop())
        table.append(row[:width] + [-1] * (width - len(row)))
        for t in range(past[i]):
            for x in (k, v):
                if t >= prefix or i == 0:
                    x[row[t // BLOCK], :, t % BLOCK] = torch.randn(kv_heads, dim, generator=g)
    k, v = k.to(dtype).cuda(), v.to(dtype).cuda()
    qkv = torch.randn(rows, heads + 2 * kv_heads, dim, generator=g).to(dtype).cuda()
    cache = rs.KVCache(k, v)
    groups = (dev([0, n]), dev([prefix])) if prefix else (None, None)
    batch = rs.KVBatch(dev(table), dev([0] * (n + 1)), dev([0] * n), rows, *groups)
    pos, slots, counts = dev([0] * rows), dev([0] * rows, torch.int64), dev([0, 0], torch.int64)
    rs.kv_tables(ctx.h, batch, dev(new), dev(past), dev([shared]) if prefix else None, dev(rest), pos, slots, counts)
    rs.kv_append(ctx.h, cache, qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:], slots)
    out, lse = torch.full((rows, heads, dim), 7.0, dtype=dtype, device="cuda"), torch.full((rows, heads), 7.0, device="cuda")
    rs.kv_attend(ctx.h, cache, batch, qkv[:, :heads], dim ** -0.5, out, lse)
    assert counts.tolist()[1] == sum(new) > rows
    s = Chain()
    # the definition has a row's keys from its position: the request ends for it with its last row
    s.q, s.k, s.v, s.table, s.scale = qkv[:, :heads].cpu(), k.cpu(), v.cpu(), batch.tensors[0].cpu(), dim ** -0.5
    s.q_start, s.kv_len = [0], []
    for a, b in zip(new, past):
        here = min(a, rows - s.q_start[-1])
        s.q_start.append(s.q_start[-1] + here)
        s.kv_len.append(b + here if here else 0)
    assert pos.tolist() == [b + t for b, a, e in zip(past, s.q_start, s.q_start[1:]) for t in range(e - a)]
    compare(s, out, lse)


@pytest.mark.parametrize("heads,kv_heads,dim,dtype", [(8, 2, 128, BF), (4, 4, 64, torch.float16), (7, 1, 64, BF)])
@pytest.mark.parametrize("prefix", [0, 96])
@pytest.mark.parametrize("new,past,rows", [([10], [100], 4), ([1, 10, 3], [96, 100, 130], 5), ([3, 400], [128, 160], 203), ([2, 300, 5], [96, 99, 97], 130),
                                           ([40] * 5, [96, 111, 128, 200, 97], 99)])
def test_rows_see_what_stands_before_them(ctx, heads, kv_heads, dim, dtype, prefix, new, past, rows):  # noqa: F811
    cut_step(ctx, 41, new, past, rows, heads, kv_heads, dim, dtype, prefix)


def test_rows_that_end_in_the_first_request_or_among_many(ctx):  # noqa: F811
    cut_step(ctx, 42, [90, 60], [0, 0], 37, 8, 2, 64, BF)
    cut_step(ctx, 43, [5] * 300 + [200], [64] * 301, 1600, 2, 1, 64, BF, 64)   # more jobs than a CTA plans for itself
