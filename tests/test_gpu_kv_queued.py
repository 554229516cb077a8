"""Steps queued behind one another: each kernel begins before the one ahead of it has ended, and reads what that writes."""
import random

import pytest

from kv_reference import BLOCK, ref_tables
from paper_2606_17081_gb300 import routesim as rs

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

BF = torch.bfloat16


@pytest.fixture(scope="module")
def ctx():
    c = rs.Context(W=1, K=1024)
    yield c
    c.close()


def test_steps_that_follow_one_another_without_a_wait(ctx):
    """Sixty steps queued at once on the same buffers, each writing what the next one reads, and the tensors of a step
    written by the stream just before it."""
    r = random.Random(44)
    dev = lambda x, t=torch.int32: torch.tensor(x, dtype=t, device="cuda")  # noqa: E731
    n, heads, dim, width, blocks, rows = 40, 2, 64, 40, 40 * 40, 400
    k, v = (torch.zeros(blocks, heads, BLOCK, dim, dtype=BF, device="cuda") for _ in range(2))
    cache = rs.KVCache(k, v)
    table, q_start, kv_len, q_len, prev = dev([[-1] * width] * n), dev([0] * (n + 1)), dev([0] * n), dev([0] * n), dev([0] * n)
    free, slots, pos, counts = dev([0] * blocks), dev([0] * rows, torch.int64), dev([0] * rows), dev([0, 0], torch.int64)
    batch = rs.KVBatch(table, q_start, kv_len, rows)
    new = [[r.choice([0, 1, 1, 1, 7]) for _ in range(n)] for _ in range(60)]
    past, used, want_table, seen, want = [0] * n, 0, [[-1] * width] * n, [], []
    rows_of = [torch.randn(rows, 2 * heads, dim, device="cuda").to(BF) for _ in new]
    steps = []
    for q in new:
        steps.append((dev(q), dev(past), dev([(used + j) % blocks for j in range(blocks)])))
        want_table, starts, lens, p, s, c = ref_tables(q, past, want_table, [(used + j) % blocks for j in range(blocks)], rows)
        want.append((starts, lens, p, s, c))
        used += c[0]
        past = lens
    torch.cuda.synchronize()
    for (a, b, f), x in zip(steps, rows_of):
        q_len.copy_(a)
        prev.copy_(b)
        free.copy_(f)
        rs.kv_tables(ctx.h, batch, q_len, prev, None, free, pos, slots, counts)
        rs.kv_append(ctx.h, cache, x[:, :heads], x[:, heads:], slots)
        seen.append([t.clone() for t in (q_start, kv_len, pos, slots, counts)])
    for got, exp in zip(seen, want):
        assert [t.tolist() for t in got] == list(exp)
    assert table.tolist() == want_table
    wk, wv = torch.zeros_like(k), torch.zeros_like(v)
    for (_, _, _, s, _), x in zip(want, rows_of):
        at = torch.tensor([i for i, y in enumerate(s) if y >= 0], device="cuda")
        y = torch.tensor([y for y in s if y >= 0], device="cuda")
        wk[y // BLOCK, :, y % BLOCK], wv[y // BLOCK, :, y % BLOCK] = x[at, :heads], x[at, heads:]
    assert torch.equal(k, wk) and torch.equal(v, wv)
