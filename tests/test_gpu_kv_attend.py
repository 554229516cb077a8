"""kv_attend against the definition in 64 bits.

Tolerances, from the types alone (u = 2^-8 in bf16, 2^-11 in fp16, the half step
of a rounding): every weight p_j is rounded once before the product with V, so
the quotient is off by at most u sum p_j |v_j| / sum p_j =: u A; out is rounded
once, u |out|.  Sums and scores in 32 bits: 2^-14 A covers the scores' error
(some 2^-20 of sum |q_d k_d|, here below 2^6 after scaling).  fp16 weights below
2^-14 keep an absolute step of 2^-25 of the largest: 2^-25 keys max |v|.
lse: the scores' error again, 2^-14, and 2^-20 of its size."""
import random

import pytest

from kv_reference import BLOCK, Step, ref_attend
from paper_2606_17081_gb300 import routesim as rs

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def ctx():
    c = rs.Context(W=1, K=1024)
    yield c
    torch.cuda.synchronize()
    attend(c, Step(0, [1], [3], 1, 1, 64, BF))   # (would report a wait that ran out in a call before)
    c.close()


def attend(ctx, s, out=None, q=None):
    cache, batch, qd = s.to(rs)
    q = qd if q is None else q
    out = torch.full_like(qd, 7.0) if out is None else out
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    rs.kv_attend(ctx.h, cache, batch, q, s.scale, out, lse)
    return out, lse


def compare(s, out, lse, n_keys=None):
    want, want_lse = s.expected()
    wide, _ = ref_attend(s.q, s.k, s.v.abs(), s.table.tolist(), s.q_start, s.kv_len, s.scale)   # A
    u = 2.0 ** -8 if s.q.dtype == BF else 2.0 ** -11
    tol = u * (wide + want.abs()) * 1.01 + 2.0 ** -14 * wide + 1e-7
    if s.q.dtype == HF:
        tol = tol + 2.0 ** -25 * max(s.kv_len + [0]) * 6.0
    got = out.cpu().double()
    assert torch.isfinite(got).all()
    over = (got - want).abs() - tol
    assert (over <= 0).all(), f"{over.max().item()} past the bound at {torch.nonzero(over > 0)[:4].tolist()}"
    gl = lse.cpu().double()
    none = torch.isinf(want_lse)
    assert torch.equal(torch.isinf(gl) & (gl < 0), none)
    assert (got[none] == 0).all()
    assert ((gl - want_lse)[~none].abs() <= 2.0 ** -14 + 2.0 ** -20 * want_lse[~none].abs()).all()


HEADS = [(4, 4, 64), (8, 2, 128), (7, 1, 128), (12, 4, 64), (40, 1, 64), (128, 1, 128), (6, 2, 128), (1, 1, 64), (48, 16, 64)]


@pytest.mark.parametrize("heads,kv_heads,dim", HEADS)
@pytest.mark.parametrize("dtype", [BF, HF])
def test_single_tokens(ctx, heads, kv_heads, dim, dtype):
    """Contexts around blocks' and tiles' ends, an empty one, a request without tokens, rows of none."""
    lens = [1, 2, 15, 16, 17, 64, 127, 128, 129, 0, 255, 256, 257, 511, 300]
    new = [1 if x else 0 for x in lens]
    s = Step(1, new, [x - q for x, q in zip(lens, new)], heads, kv_heads, dim, dtype, pad=3)
    compare(s, *attend(ctx, s))


@pytest.mark.parametrize("heads,kv_heads,dim", HEADS)
@pytest.mark.parametrize("order", ["heads", "tokens"])
def test_shared_prefixes(ctx, heads, kv_heads, dim, order):
    r = random.Random(heads)
    n = 23
    new = [r.choice([0, 1, 1, 1, 2, 5]) for _ in range(n)]
    start, prefix = [1, 9, 9, 20, 22], [320, 48, 512, 16]
    ctxs = [r.randint(0, 200) for _ in range(n)]
    for g in range(4):
        for i in range(start[g], start[g + 1]):
            ctxs[i] += prefix[g]
    s = Step(2, new, ctxs, heads, kv_heads, dim, BF, start, prefix, pad=2, order=order)
    compare(s, *attend(ctx, s))


def test_members_that_end_inside_the_prefix(ctx):
    """Short contexts, empty ones and prompts that still write the prefix itself, beside full members."""
    prefix = [400]
    ctxs = [400, 0, 77, 390, 500, 399, 400, 130, 0, 401] + [400 + i for i in range(12)]
    new = [1, 1, 3, 20, 1, 1, 0, 40, 0, 2] + [1] * 12
    for heads, kv_heads, dim in ((8, 2, 128), (16, 16, 64), (5, 1, 64)):
        s = Step(3, new, ctxs, heads, kv_heads, dim, BF, [0, len(new)], prefix, pad=1)
        compare(s, *attend(ctx, s))


def test_rows_before_the_first_position(ctx):
    """More new tokens than the context holds: the first rows see nothing."""
    s = Step(4, [6, 1, 200], [0, 3, 0], 8, 2, 64, BF)
    s.kv_len = [2, 4, 70]
    s.kv_len[1] = 0
    compare(s, *attend(ctx, s))


@pytest.mark.parametrize("heads,kv_heads,dim,dtype", [(8, 2, 128, BF), (4, 4, 64, HF), (7, 1, 128, BF), (24, 8, 64, BF), (128, 1, 64, BF)])
@pytest.mark.parametrize("new,ctxs", [([300], [0]), ([128, 129, 1, 127], [0, 5, 900, 128]), ([513], [1000]), ([65, 700, 2], [16, 333, 2000])])
def test_prompts(ctx, heads, kv_heads, dim, dtype, new, ctxs):
    s = Step(5, new, ctxs, heads, kv_heads, dim, dtype, pad=1)
    compare(s, *attend(ctx, s))


def test_prompts_with_a_shared_prefix(ctx):
    s = Step(6, [100, 3, 260, 1, 40], [256, 256, 300, 256, 999], 8, 2, 128, BF, [0, 4], [256])
    compare(s, *attend(ctx, s))


@pytest.mark.parametrize("n,heads,kv_heads,prefix,own", [(1, 8, 1, 0, 9000), (2, 4, 4, 0, 5000), (40, 16, 2, 6000, 40), (3, 32, 8, 2048, 3000)])
def test_long_contexts_are_split_and_joined(ctx, n, heads, kv_heads, prefix, own):
    r = random.Random(own)
    ctxs = [prefix + r.randint(own // 2, own) for _ in range(n)]
    s = Step(7, [1] * n, ctxs, heads, kv_heads, 64, BF, [0, n], [prefix])
    compare(s, *attend(ctx, s))


@pytest.mark.parametrize("growth", [1.0, 40.0, -40.0])
@pytest.mark.parametrize("heads,new", [(8, 1), (2, 150)])
def test_scores_that_grow_along_the_keys(ctx, growth, heads, new):
    """The running maximum moves in every tile (or in the first alone), by far more than the weights' range."""
    n = 1200
    s = Step(8, [new], [n - new], heads, 2, 64, BF)
    ramp = torch.linspace(0, growth, n)
    for j in range(n):
        b = int(s.table[0, j // BLOCK])
        s.k[b, :, j % BLOCK, 0] = ramp[j].to(BF)
    s.q[:, :, 0] = 8.0
    s.q[:, :, 1:] *= 0.25
    compare(s, *attend(ctx, s))


@pytest.mark.parametrize("growth", [1.0, 40.0, -40.0])
def test_scores_that_grow_in_fp16(ctx, growth):
    """Weights stay within fp16's range although the running maximum starts far below."""
    n = 700
    s = Step(18, [1, 90], [n - 1, n - 90], 4, 2, 64, HF)
    for i in range(2):
        for j in range(n):
            s.k[int(s.table[i, j // BLOCK]), :, j % BLOCK, 0] = growth * j / n
    s.q[:, :, 0] = 6.0
    s.q[:, :, 1:] *= 0.25
    compare(s, *attend(ctx, s))


@pytest.mark.parametrize("heads,kv_heads,dim", [(8, 2, 128), (16, 16, 64), (5, 1, 64)])
def test_short_tables_are_not_cut(ctx, heads, kv_heads, dim):
    """Rows of at most 16 blocks and no groups: the jobs stay whole."""
    r = random.Random(dim)
    new = [r.choice([0, 1, 1, 3, 40]) for _ in range(70)]
    s = Step(16, new, [r.randint(0, 200) for _ in new], heads, kv_heads, dim, BF, pad=5)
    assert s.table.shape[1] <= 16
    compare(s, *attend(ctx, s))


def test_many_requests_and_groups(ctx):
    """More requests, and more groups, than a CTA plans for itself; more prefix jobs than a warp has lanes."""
    r = random.Random(17)
    for n, per, prefix in ((1100, 0, 0), (1200, 1, 32), (90, 2, 400), (1030, 10, 160)):
        starts = list(range(0, n, per)) + [n] if per else None
        new = [r.choice([0, 1, 1, 1, 2]) for _ in range(n)]
        ctxs = [prefix + r.randint(0, 40) for _ in range(n)]
        s = Step(17, new, ctxs, 2, 1, 64, BF, starts, [prefix] * (len(starts) - 1) if per else None, pad=1)
        compare(s, *attend(ctx, s))


def test_a_long_prompt_beside_single_tokens(ctx):
    """More jobs than a CTA plans for itself, with a group's prefix among them."""
    ctxs = [256] * 40 + [300]
    s = Step(19, [1] * 40 + [1100], ctxs, 128, 1, 64, BF, [0, 40], [256])
    compare(s, *attend(ctx, s))


def test_strided_and_shifted_tensors(ctx):
    """q as columns of a projection, out inside a wider buffer that stays as it was around it."""
    s = Step(9, [1, 4, 30], [50, 200, 10], 8, 2, 64, BF)
    qkv = torch.zeros(s.rows, 12 * 64, dtype=BF, device="cuda")
    q = qkv[:, 128:640].view(s.rows, 8, 64)
    q.copy_(s.q)
    wide = torch.full((s.rows, 10, 72), 3.0, dtype=BF, device="cuda")
    out, lse = attend(ctx, s, out=wide[:, 1:9, :64], q=q)
    compare(s, out, lse)
    assert (wide[:, 0] == 3).all() and (wide[:, 9] == 3).all() and (wide[:, :, 64:] == 3).all()
    turned = s.q.transpose(0, 1).contiguous().cuda().transpose(0, 1)   # head-major q
    compare(s, *attend(ctx, s, q=turned))


def test_without_lse_and_the_same_twice(ctx):
    s = Step(10, [1] * 20, [700] * 20, 8, 2, 128, BF, [0, 20], [640])
    cache, batch, q = s.to(rs)
    a, b, c = (torch.zeros_like(q) for _ in range(3))
    lse = torch.zeros(q.shape[:2], device="cuda")
    rs.kv_attend(ctx.h, cache, batch, q, s.scale, a, lse)
    rs.kv_attend(ctx.h, cache, batch, q, s.scale, b)
    rs.kv_attend(ctx.h, cache, batch, q, s.scale, c)
    assert torch.equal(a, b) and torch.equal(a, c)
    compare(s, a, lse)


def test_blocks_outside_the_cache_read_as_zeros(ctx):
    s = Step(11, [1, 3], [200, 90], 4, 2, 64, BF)
    s.table[0, 2], s.table[1, 0] = -1, s.n_blocks + 9
    out, lse = attend(ctx, s)
    zero = torch.zeros(2, *s.k.shape[1:], dtype=BF)
    s.k, s.v = torch.cat([s.k, zero]), torch.cat([s.v, zero])
    s.table[0, 2] = s.table[1, 0] = s.n_blocks
    compare(s, out, lse)


def test_offsets_past_32_bits(ctx):
    """Blocks past 2^31 elements of a cache."""
    blocks = (1 << 21) + 200
    s = Step(12, [1, 5], [300, 77], 4, 1, 64, BF)
    low = torch.randperm(s.n_blocks)
    k, v = (torch.empty(blocks, 1, BLOCK, 64, dtype=BF, device="cuda") for _ in range(2))
    at = blocks - 1 - low
    k[at.cuda()], v[at.cuda()] = s.k.cuda(), s.v.cuda()
    table = torch.where(s.table >= 0, at[s.table.clamp(min=0).long()].int(), s.table)
    _, batch, q = s.to(rs)
    moved = rs.KVBatch(table.cuda(), batch.tensors[1], batch.tensors[2], s.rows)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    rs.kv_attend(ctx.h, rs.KVCache(k, v), moved, q, s.scale, out, lse)
    compare(s, out, lse)


def test_lengths_that_do_not_fit_together_stay_inside_the_arrays(ctx):
    """Starts that decrease or pass the rows, lengths past the table: rows may hold anything, the guard around out may not."""
    s = Step(13, [2, 3, 4], [40, 50, 60], 4, 2, 64, BF)
    cache, batch, q = s.to(rs)
    for q_start, kv_len, start, prefix in (([0, 5, 2, 9], [42, 53, 64], None, None), ([0, 2, 5, 100], [42, 53, 64], None, None),
                                           ([-4, 2, 5, 9], [42, -3, 64], None, None), ([0, 2, 5, 9], [10 ** 9, 53, 2 ** 31 - 1], None, None),
                                           ([0, 2, 5, 9], [42, 53, 64], [0, 3], [2 ** 31 - 1]), ([0, 2, 5, 9], [42, 53, 64], [2, 1], [32]),
                                           ([0, 2, 5, 9], [42, 53, 64], [-3, 90], [32])):
        dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        b = rs.KVBatch(batch.tensors[0], dev(q_start), dev(kv_len), s.rows, dev(start) if start else None, dev(prefix) if start else None)
        guard = torch.full((s.rows + 40, 4, 64), 3.0, dtype=BF, device="cuda")
        lse = torch.full((s.rows + 40, 4), 3.0, device="cuda")
        rs.kv_attend(ctx.h, cache, b, q, s.scale, guard[20:20 + s.rows], lse[20:20 + s.rows])
        torch.cuda.synchronize()
        for x in (guard, lse):
            assert (x[:20] == 3).all() and (x[20 + s.rows:] == 3).all()


def test_no_request_at_all(ctx):
    s = Step(14, [1], [9], 4, 2, 64, BF)
    cache, _, _ = s.to(rs)
    z = torch.zeros(0, dtype=torch.int32, device="cuda")
    b = rs.KVBatch(z.reshape(0, 3), torch.zeros(1, dtype=torch.int32, device="cuda"), z, 5)
    q = torch.ones(5, 4, 64, dtype=BF, device="cuda")
    out, lse = torch.ones_like(q), torch.ones(5, 4, device="cuda")
    rs.kv_attend(ctx.h, cache, b, q, 1.0, out, lse)
    assert (out == 0).all() and (lse == -float("inf")).all()


def test_on_another_stream_and_in_a_graph():
    """tables, append and attend captured as one step and replayed on new lengths."""
    st = torch.cuda.Stream()
    c = rs.Context(W=1, K=1024, stream=st.cuda_stream)
    n, heads, kv_heads, dim, width = 6, 8, 2, 64, 40
    dev = lambda x, t=torch.int32: torch.tensor(x, dtype=t, device="cuda")  # noqa: E731
    k, v = (torch.full((300, kv_heads, BLOCK, dim), float("nan"), dtype=BF, device="cuda") for _ in range(2))
    table, q_start, kv_len = dev([[-1] * width] * n), dev([0] * (n + 1)), dev([0] * n)
    prev, q_len, free = dev([0] * n), dev([1] * n), dev(list(range(300)))
    rows = 64
    batch, cache = rs.KVBatch(table, q_start, kv_len, rows), rs.KVCache(k, v)
    pos, slots, counts = dev([0] * rows), dev([0] * rows, torch.int64), dev([0, 0], torch.int64)
    qkv = torch.randn(rows, heads + 2 * kv_heads, dim, device="cuda").to(BF)
    out, lse = torch.empty(rows, heads, dim, dtype=BF, device="cuda"), torch.empty(rows, heads, device="cuda")

    def step():
        rs.kv_tables(c.h, batch, q_len, prev, None, free, pos, slots, counts)
        rs.kv_append(c.h, cache, qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:], slots)
        rs.kv_attend(c.h, cache, batch, qkv[:, :heads], dim ** -0.5, out, lse)

    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        step()
    st.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        step()
    past, used = [0] * n, 0
    for lens in ([9, 1, 20, 0, 16, 17], [1, 1, 1, 1, 1, 1], [1, 30, 1, 1, 0, 1]):
        q_len.copy_(dev(lens))
        prev.copy_(dev(past))
        qkv.copy_(torch.randn(rows, heads + 2 * kv_heads, dim, device="cuda").to(BF))
        free.copy_(dev([x % 300 for x in range(used, used + 300)]))
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            g.replay()
        st.synchronize()
        used += int(counts[0])
        past = [a + b for a, b in zip(past, lens)]
        s = Step.__new__(Step)
        s.q, s.k, s.v, s.table = qkv[:, :heads].cpu(), k.cpu(), v.cpu(), table.cpu()
        s.q_start, s.kv_len, s.scale = q_start.tolist(), kv_len.tolist(), dim ** -0.5
        assert s.kv_len == past and s.q_start[-1] == sum(lens)
        compare(s, out, lse)
    c.close()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_many_rows_of_many_parts(ctx, dim, dtype):
    """9600 rows to join, a prefix's jobs over seven CTAs or so each, own parts of one tile."""
    s = Step(23, [149, 0, 151], [4100, 4096, 4111], 16, 4, dim, dtype, group_start=[0, 3], prefix=[4096])
    compare(s, *attend(ctx, s))


def test_a_capture_keeps_its_workspace():
    """A capture that would have to allocate is refused; a captured step replays after larger calls."""
    st = torch.cuda.Stream()
    c = rs.Context(W=1, K=1024, stream=st.cuda_stream)
    small, large = Step(21, [1, 2], [40, 300], 8, 2, 64, BF), Step(22, [400, 3], [900, 2000], 16, 4, 128, BF)
    (cache, batch, q), big = small.to(rs), large.to(rs)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    out2, lse2 = torch.empty_like(big[2]), torch.empty(big[2].shape[:2], device="cuda")
    torch.cuda.synchronize()

    def refused(cache, batch, q, out, lse):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=st):
            with pytest.raises(rs.RoutesimError) as e:
                rs.kv_attend(c.h, cache, batch, q, small.scale, out, lse)
        assert e.value.status == rs.RS_ERR_STATE

    refused(cache, batch, q, out, lse)
    with torch.cuda.stream(st):
        rs.kv_attend(c.h, cache, batch, q, small.scale, out, lse)
    st.synchronize()
    refused(*big, out2, lse2)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        rs.kv_attend(c.h, cache, batch, q, small.scale, out, lse)
    with torch.cuda.stream(st):
        rs.kv_attend(c.h, *big, large.scale, out2, lse2)
    fill = [torch.full((1 << 22,), float("nan"), device="cuda") for _ in range(8)]   # (what a freed workspace could become)
    for _ in range(2):
        out.fill_(7)
        lse.fill_(7)
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            g.replay()
            rs.kv_attend(c.h, *big, large.scale, out2, lse2)
        st.synchronize()
        compare(small, out, lse)
        compare(large, out2, lse2)
    assert all(bool(x.isnan().all()) for x in fill)
    c.close()


def test_refusals(ctx):
    s = Step(15, [1], [9], 4, 2, 64, BF)
    cache, batch, q = s.to(rs)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    for bad in (dict(q=q.half()), dict(out=out.float()), dict(q=q.cpu()), dict(q=q[:, :, :32]), dict(lse=lse.double()), dict(lse=lse[:, :2]),
                dict(q=torch.cat([q, q])), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
                dict(q=q[:, :3], out=out[:, :3], lse=None)):
        a = dict(q=q, scale=0.1, out=out, lse=lse)
        a.update(bad)
        with pytest.raises(rs.RoutesimError) as e:
            rs.kv_attend(ctx.h, cache, batch, a["q"], a["scale"], a["out"], a["lse"])
        assert e.value.status == rs.RS_ERR_INVALID
    L = rs.lib()
    two = torch.zeros(4, 8, 64, dtype=BF, device="cuda")
    b2 = rs.KVBatch(batch.tensors[0], batch.tensors[1], batch.tensors[2], 4)

    def call(q=two.data_ptr(), heads=8, ts=512, hs=64, out=two.data_ptr(), cache=cache, batch=b2):
        return L.kv_attend(ctx.h, cache.ref, batch.ref, q, heads, ts, hs, 1.0, out, 512, 64, None)

    assert call(q=two.data_ptr() + 2) == call(q=None) == call(out=None) == call(ts=508) == call(hs=0) == call(hs=-64) == rs.RS_ERR_INVALID
    assert call(heads=0) == call(heads=7) == call(heads=258) == rs.RS_ERR_INVALID
    assert rs.route_last_error(ctx.h)
    bad = rs.KVCache(cache.k, cache.v)
    bad.desc.head_dim = 80
    assert call(cache=bad) == rs.RS_ERR_INVALID
    none = rs.KVBatch(batch.tensors[0], batch.tensors[1], batch.tensors[2], 0)
    assert call(batch=none) == rs.RS_OK
