"""kv_attend4 on starts and lengths that do not fit together, in steps of every size (bounds: kv4_reference.compare)."""
import pytest

from kv4_reference import Step4, compare, empty_cache
from paper_2606_17081_gb300 import routesim as rs

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

from test_gpu_kv4_attend import BF, HF, attend, ctx  # noqa: E402, F401


@pytest.mark.parametrize("heads,kv_heads,dim,dtype", [(4, 2, 64, BF), (8, 2, 128, HF)])
@pytest.mark.parametrize("new,ctxs,groups", [([1, 2, 0, 1], [300, 40, 5, 17], None), ([1] * 3, [700, 900, 130], ([0, 3], [128])),
                                             ([70, 2, 1], [300, 40, 1000], None), ([1] * 40, [60 + 9 * i for i in range(40)], ([2, 30], [48]))])
def test_a_first_start_past_row_0(ctx, heads, kv_heads, dim, dtype, new, ctxs, groups):  # noqa: F811
    """The rows before it belong to no request, whatever a call before, with parts of every kind, left in the workspace."""
    before = Step4(71, [90] * 4, [2000] * 4, 16, 2, 128, BF, [0, 4], [1024])
    attend(ctx, before)
    s = Step4(72, new, ctxs, heads, kv_heads, dim, dtype, *(groups or ()), pad=7)
    s.q_start = [x + 5 for x in s.q_start]
    compare(s, *attend(ctx, s))


SIZES = [([30, 40, 20], [400, 50, 600], 8, 2, 64, BF), ([30, 300, 20], [4000, 50, 600], 8, 2, 128, BF), ([1] * 40, [60 + 9 * i for i in range(40)], 4, 4, 64, HF),
         ([1, 2, 1, 0] * 12, [900 - 11 * i for i in range(48)], 14, 2, 128, BF), ([1] * 6, [40, 900, 33, 70, 200, 5], 4, 2, 64, BF)]


def odd_lengths(n, rows, starts, lens):
    """(starts, lengths, first requests of groups, prefixes) of n requests that no step should have."""
    some = [0, 1, n // 2, n]
    yield starts, [2 ** 31 - 1] * n, None, None
    yield starts, [-5 if i % 2 else x for i, x in enumerate(lens)], some, [64, 32, 2 ** 31 - 1]
    yield [x + rows // 3 for x in starts], lens, None, None
    yield [x + rows // 3 for x in starts], lens, [0, n], [48]
    yield [x - rows // 3 for x in starts], lens, some, [16, 0, 4096]
    yield [rows - x for x in starts], lens, None, None
    yield [rows - x for x in starts], lens, [0, n], [48]
    yield [0 if i % 2 else rows for i in range(n + 1)], lens, None, None   # (more rows than there is room for)
    yield [0 if i % 2 else rows for i in range(n + 1)], lens, [0, n // 2, n], [48, 64]
    yield [(7 * i * i) % (rows + 9) - 3 for i in range(n + 1)], lens, [n // 2, 1, n + 5], [32, 400]
    yield [0] + [2 ** 31 - 1] * n, lens, [0, n], [128]
    yield [-2 ** 31] * n + [2 ** 31 - 1], lens, [-9, 2 ** 31 - 1], [32]
    yield [rows] * (n + 1), lens, [n, n], [32]
    yield starts, lens, [0, n, 0, n], [256, 32, 2 ** 31 - 16]


@pytest.mark.parametrize("new,ctxs,heads,kv_heads,dim,dtype", SIZES)
def test_lengths_that_do_not_fit_together_stay_inside_the_arrays(ctx, new, ctxs, heads, kv_heads, dim, dtype):  # noqa: F811
    """Rows may hold anything, the guard around out and lse may not, and a step that fits comes out right behind them."""
    s = Step4(73, new, ctxs, heads, kv_heads, dim, dtype, pad=3)
    cache, batch, q = s.to(rs)
    table = batch.tensors[0].clone()
    table[-1, 0], table[0, -1] = 2 ** 31 - 1, -2 ** 31
    n = len(new)
    for starts, lens, first, prefix in odd_lengths(n, s.rows, s.q_start, s.kv_len):
        if prefix and len(prefix) > n:
            continue
        dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        b = rs.KVBatch(table, dev(starts), dev(lens), s.rows, dev(first) if first else None, dev(prefix) if prefix else None)
        guard = torch.full((s.rows + 40, heads, dim), 3.0, dtype=dtype, device="cuda")
        lse = torch.full((s.rows + 40, heads), 3.0, device="cuda")
        rs.kv_attend4(ctx.h, cache, b, q, s.scale, guard[20:20 + s.rows], lse[20:20 + s.rows])
        torch.cuda.synchronize()
        for x in (guard, lse):
            assert (x[:20] == 3).all() and (x[20 + s.rows:] == 3).all()
        rs.kv_status(ctx.h)
        again, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        rs.kv_attend4(ctx.h, cache, batch, q, s.scale, again, lse)
    compare(s, again, lse)


@pytest.mark.parametrize("rows", [1, 5, 40, 700])
def test_no_request_in_steps_of_every_size(ctx, rows):  # noqa: F811
    cache = empty_cache(rs, 4, 2, 64)
    z = torch.zeros(0, dtype=torch.int32, device="cuda")
    b = rs.KVBatch(z.reshape(0, 3), torch.zeros(1, dtype=torch.int32, device="cuda"), z, rows)
    q = torch.ones(rows, 16, 64, dtype=BF, device="cuda")
    out, lse = torch.ones_like(q), torch.ones(rows, 16, device="cuda")
    rs.kv_attend4(ctx.h, cache, b, q, 1.0, out, lse)
    assert (out == 0).all() and (lse == -float("inf")).all()
