"""kv_tables and kv_append against plain Python: equal to the last bit."""
import random

import pytest

from kv_reference import BLOCK, ref_tables
from paper_2606_17081_gb300 import routesim as rs

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)


@pytest.fixture(scope="module")
def ctx():
    c = rs.Context(W=1, K=1024)
    yield c
    c.close()


def dev(x, dtype=None):
    return torch.tensor(x, dtype=dtype or torch.int32, device="cuda")


def run(ctx, q, c, table, free, rows, group_start=None, prefix=None, lists=None):
    t = dev(table).reshape(len(q), -1)
    n = len(q)
    q_start, kv_len = torch.full((n + 1,), 77, dtype=torch.int32, device="cuda"), torch.full((n,), 77, dtype=torch.int32, device="cuda")
    b = rs.KVBatch(t, q_start, kv_len, rows, dev(group_start) if prefix else None, dev(prefix) if prefix else None)
    pos, slots = torch.full((rows,), 77, dtype=torch.int32, device="cuda"), torch.full((rows,), 77, dtype=torch.int64, device="cuda")
    counts = torch.full((2,), 77, dtype=torch.int64, device="cuda")
    width = max((len(x) for x in lists), default=0) if prefix else 0
    pb = dev([list(x) + [-5] * (width - len(x)) for x in lists]).reshape(len(prefix), width) if prefix else None
    rs.kv_tables(ctx.h, b, dev(q), dev(c), pb, dev(free), pos, slots, counts)
    return [x.tolist() for x in (t, q_start, kv_len, pos, slots, counts)]


def check(ctx, q, c, width, free, rows, group_start=None, prefix=None, lists=None, seed=0):
    r = random.Random(seed)
    table = [[r.randrange(100000, 200000) for _ in range(width)] for _ in q]
    # (the reference pads a group's list to the longest one, as the call does)
    longest = max((len(x) for x in lists or []), default=0)
    padded = [list(x) + [-5] * (longest - len(x)) for x in lists or []]
    want = ref_tables(q, c, table, free, rows, group_start, prefix, padded)
    got = run(ctx, q, c, table, free, rows, group_start, prefix, lists)
    for name, g, w in zip(("table", "q_start", "kv_len", "positions", "slots", "counts"), got, want):
        assert g == w, name


@pytest.mark.parametrize("q,c", [([1], [0]), ([0], [0]), ([1], [15]), ([1], [16]), ([2], [15]), ([17], [0]),
                                 ([16, 1, 0, 33], [0, 16, 5, 31]), ([0, 0, 0, 1], [0, 3, 16, 15])])
def test_few_requests(ctx, q, c):
    check(ctx, q, c, 8, list(range(500, 560)), sum(q) + 2)


@pytest.mark.parametrize("n,seed", [(1, 1), (31, 2), (513, 3), (1024, 4), (3001, 5)])
def test_many_requests_in_groups(ctx, n, seed):
    r = random.Random(seed)
    q = [r.choice([0, 1, 1, r.randint(0, 70)]) for _ in range(n)]
    groups = r.randint(1, min(n, 40))
    start = sorted(r.randint(0, n) for _ in range(groups + 1))
    prefix = [r.randint(0, 400) for _ in range(groups)]
    lists = [[r.randrange(1000) for _ in range(p // BLOCK)] for p in prefix]
    c = [r.randint(0, 600) for _ in range(n)]   # (some inside their group's prefix)
    need = sum(-(-(a + b) // BLOCK) for a, b in zip(q, c))
    for free_n, width, rows in ((need, 60, sum(q) + 5), (need // 3, 60, sum(q)), (need, 20, sum(q) // 2)):
        check(ctx, q, c, width, [5000 + k for k in range(free_n)], rows, start, prefix, lists, seed)


def test_more_groups_than_shared_memory_keeps(ctx):
    n = 2500
    check(ctx, [1] * n, [33 + i % 40 for i in range(n)], 8, list(range(9000, 9000 + n)), n,
          list(range(n + 1)), [32] * n, [[i, i + 1] for i in range(n)])


def test_the_longest_batch_and_a_long_request(ctx):
    n = 16384
    check(ctx, [1] * n, [i % 64 for i in range(n)], 8, list(range(n)), n)
    check(ctx, [3, 5000, 1], [0, 100000, 7], 8000, list(range(10 ** 6, 10 ** 6 + 400)), 5004)


def test_no_requests_and_no_free_blocks(ctx):
    b = rs.KVBatch(dev([]).reshape(0, 4), dev([9]), dev([]), 3)
    pos, slots, counts = dev([5] * 3), dev([5] * 3, torch.int64), dev([5, 5], torch.int64)
    rs.kv_tables(ctx.h, b, dev([]), dev([]), None, dev([]), pos, slots, counts)
    assert pos.tolist() == [-1] * 3 and slots.tolist() == [-1] * 3 and counts.tolist() == [0, 0]
    assert b.tensors[1].tolist() == [0]
    check(ctx, [1, 20], [16, 16], 4, [], 21)


def test_values_outside_their_range_stay_inside_the_arrays(ctx):
    """Negative lengths count as none, huge ones end at 2^31 - 17 and are cut at the table's row."""
    t = dev([[7] * 4] * 3)
    b = rs.KVBatch(t, dev([0] * 4), dev([0] * 3), 6, dev([0, 3]), dev([2 ** 31 - 1]))
    pos, slots, counts = dev([9] * 6), dev([9] * 6, torch.int64), dev([0, 0], torch.int64)
    rs.kv_tables(ctx.h, b, dev([-5, 2, 2 ** 31 - 1]), dev([-1, 2 ** 31 - 1, 2 ** 31 - 20]), dev([[1, 2]]), dev([3]), pos, slots, counts)
    assert b.tensors[1].tolist() == [0, 0, 0, 3]
    assert b.tensors[2].tolist() == [0, 2 ** 31 - 17, 2 ** 31 - 17]
    assert pos.tolist() == [2 ** 31 - 20, 2 ** 31 - 19, 2 ** 31 - 18, -1, -1, -1]
    assert slots.tolist() == [-1] * 6 and counts.tolist() == [0, 3]
    assert t.tolist() == [[1, 2, 7, 7]] * 3


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("heads,dim,n,order,shift", [(1, 64, 1, "heads", 0), (3, 128, 37, "tokens", 0), (8, 128, 1000, "heads", 0),
                                                     (2, 64, 33, "heads", 1), (2, 128, 9, "tokens", 3), (1, 128, 5, "heads", 0)])
def test_append(ctx, dtype, heads, dim, n, order, shift):
    """shift: rows that start off a 16-byte boundary."""
    blocks = n // BLOCK + 4
    shape = (blocks, 2, heads, BLOCK, dim) if order == "heads" else (blocks, 2, BLOCK, heads, dim)
    both = torch.randn(shape, device="cuda").to(dtype)
    k, v = both[:, 0], both[:, 1]
    if order == "tokens":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    flat = torch.randn(n * (2 * heads + 1) * dim + 8, device="cuda").to(dtype)
    rows = flat[shift:shift + n * (2 * heads + 1) * dim].view(n, 2 * heads + 1, dim)
    kn, vn = rows[:, :heads], rows[:, heads:2 * heads]
    slots = torch.randperm(blocks * BLOCK, device="cuda")[:n]
    slots[n // 2] = -1
    if n > 4:
        slots[1], slots[3] = blocks * BLOCK, -2 ** 40   # outside the cache: left out
    want_k, want_v = k.clone(), v.clone()
    for r, s in enumerate(slots.tolist()):
        if 0 <= s < blocks * BLOCK:
            want_k[s // BLOCK, :, s % BLOCK], want_v[s // BLOCK, :, s % BLOCK] = kn[r], vn[r]
    rs.kv_append(ctx.h, rs.KVCache(k, v), kn, vn, slots)
    assert torch.equal(k, want_k) and torch.equal(v, want_v)


def test_append_past_32_bits(ctx):
    blocks = (1 << 21) + 5   # of 1024 elements: the last lie past 2^31
    k, v = (torch.empty(blocks, 1, BLOCK, 64, dtype=torch.float16, device="cuda") for _ in range(2))
    rows = torch.randn(3, 1, 64, device="cuda").half()
    slots = dev([blocks * BLOCK - 1, (1 << 21) * BLOCK, 4], torch.int64)
    rs.kv_append(ctx.h, rs.KVCache(k, v), rows, rows, slots)
    for r, s in enumerate(slots.tolist()):
        assert torch.equal(k[s // BLOCK, 0, s % BLOCK], rows[r, 0]) and torch.equal(v[s // BLOCK, 0, s % BLOCK], rows[r, 0])


def test_refusals(ctx):
    t = dev([[1, 2]])
    b = rs.KVBatch(t, dev([0, 1]), dev([1]), 1)
    one, long, two = dev([1]), dev([1], torch.int64), dev([1, 1], torch.int64)
    rs.kv_tables(ctx.h, b, one, one, None, one, dev([0]), long, two)
    for args in ((long, one, None, one, one, long, two), (one, dev([1, 1]), None, one, one, long, two),
                 (one, one, None, long, one, long, two), (one, one, None, one, dev([0, 0]), long, two),
                 (one, one, None, one, one, one, two), (one, one, None, one, one, long, long)):
        with pytest.raises(rs.RoutesimError) as e:
            rs.kv_tables(ctx.h, b, *args)
        assert e.value.status == rs.RS_ERR_INVALID
    with pytest.raises(rs.RoutesimError, match="go together"):
        rs.KVBatch(t, dev([0, 1]), dev([1]), 1, dev([0, 1]))
    for field, value in (("n_req", -1), ("n_req", 16385), ("n_tokens", -1), ("n_tokens", (1 << 24) + 1), ("n_groups", 2), ("n_groups", -1),
                         ("max_blocks", 0), ("table_stride", 1), ("table", None), ("q_start", None), ("kv_len", None), ("n_groups", 1)):
        bad = rs.KVBatch(t, dev([0, 1]), dev([1]), 1)
        setattr(bad.desc, field, value)
        assert rs.lib().kv_tables(ctx.h, bad.ref, one.data_ptr(), one.data_ptr(), None, 0, one.data_ptr(), 1, one.data_ptr(), long.data_ptr(),
                                  two.data_ptr()) == rs.RS_ERR_INVALID, field
        assert rs.route_last_error(ctx.h)
    L = rs.lib()
    for p in range(3):   # a NULL in place of the lengths, the free list
        a = [one.data_ptr()] * 3
        a[p] = None
        assert L.kv_tables(ctx.h, b.ref, a[0], a[1], None, 0, a[2], 1, one.data_ptr(), long.data_ptr(), two.data_ptr()) == rs.RS_ERR_INVALID
    assert L.kv_tables(ctx.h, b.ref, one.data_ptr(), one.data_ptr(), None, 0, one.data_ptr(), -1, one.data_ptr(), long.data_ptr(), two.data_ptr()) == rs.RS_ERR_INVALID
    k = torch.zeros(4, 2, BLOCK, 64, dtype=torch.bfloat16, device="cuda")
    rows = torch.zeros(1, 2, 64, dtype=torch.bfloat16, device="cuda")
    cache = rs.KVCache(k, k.clone())
    for bad_k in (rows.half(), rows[:, :1], rows[0], rows.cpu()):
        with pytest.raises(rs.RoutesimError):
            rs.kv_append(ctx.h, cache, bad_k, bad_k, long)
    with pytest.raises(rs.RoutesimError):
        rs.KVCache(k, k[:3])
    with pytest.raises(rs.RoutesimError):
        rs.KVCache(k[:, :, :8], k[:, :, :8])
    for field, value in (("k", None), ("k", k.data_ptr() + 2), ("dtype", 2), ("head_dim", 96), ("n_kv_heads", 0), ("n_kv_heads", 1025), ("n_blocks", 0),
                         ("n_blocks", (1 << 27) + 1), ("stride_block", 2044), ("stride_head", 0), ("stride_token", -64), ("stride_block", 1 << 35)):
        bad = rs.KVCache(k, k.clone())
        setattr(bad.desc, field, value)
        assert L.kv_append(ctx.h, bad.ref, rows.data_ptr(), rows.data_ptr(), 128, 64, 1, long.data_ptr()) == rs.RS_ERR_INVALID, (field, value)
    assert L.kv_append(ctx.h, cache.ref, None, rows.data_ptr(), 128, 64, 1, long.data_ptr()) == rs.RS_ERR_INVALID
    assert L.kv_append(ctx.h, cache.ref, rows.data_ptr(), rows.data_ptr(), 128, 64, -1, long.data_ptr()) == rs.RS_ERR_INVALID
    assert L.kv_append(ctx.h, cache.ref, rows.data_ptr(), rows.data_ptr(), 128, 64, 0, None) == rs.RS_OK
