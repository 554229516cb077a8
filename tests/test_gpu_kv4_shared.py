"""kv_attend4 on prefixes that are jobs of their own, whatever that saves: the tests of steps with groups, here and in
test_gpu_kv4_attend.py, once more with a build that shares every prefix that costs less so (the library's own limit leaves
most small ones to their members).  Bounds: kv4_reference.compare."""
import os
import random
import subprocess
import sys

import pytest

from kv4_reference import BLOCK, Step4, compare, empty_cache
from paper_2606_17081_gb300 import build as B
from paper_2606_17081_gb300 import routesim as rs

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

import test_gpu_kv4_attend as T  # noqa: E402
from test_gpu_kv4_attend import BF, HF, attend, ctx, step_of  # noqa: E402, F401

HERE = os.path.dirname(os.path.abspath(__file__))
SHARING = os.environ.get("KV4_SHARES") == "1"   # in the process that runs the other build
# a group of warps' rows, of a CTA's, of several CTAs'; beside a request of its own; of a prefix that the library shares too
GROUPS = [([1] * 6, [260, 300, 256, 290, 400, 257], [0, 6], [256]), ([1] * 40, [256 + 7 * i for i in range(40)], [0, 40], [256]),
          ([3] * 30 + [200], [320 + 5 * i for i in range(30)] + [40], [0, 30], [320]), ([1] * 44, [8192 + i for i in range(44)], [0, 44], [8192])]


@pytest.mark.parametrize("new,ctxs,start,prefix", GROUPS)
@pytest.mark.parametrize("dim,dtype,order", [(64, BF, "heads"), (128, HF, "tokens")])
def test_groups(ctx, new, ctxs, start, prefix, dim, dtype, order):  # noqa: F811
    """The result, the same twice, and (in the other build) not by the way that a step without groups takes."""
    s = Step4(91, new, ctxs, 8, 2, dim, dtype, start, prefix, pad=1, order=order)
    cache, batch, q = s.to(rs)
    alone = rs.KVBatch(*batch.tensors[:3], s.rows)
    got = []
    for b in (batch, batch, alone):
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        rs.kv_attend4(ctx.h, cache, b, q, s.scale, out, lse)
        compare(s, out, lse)
        got.append((out, lse))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    if SHARING:   # (the sums' order differs)
        assert not torch.equal(got[0][1], got[2][1])


@pytest.mark.parametrize("new,ctxs,start,prefix", GROUPS[1:])
@pytest.mark.parametrize("dim", [64, 128])
def test_rows_of_nan_and_of_extreme_sizes(ctx, dim, new, ctxs, start, prefix):  # noqa: F811
    T.test_rows_of_nan_and_of_extreme_sizes(ctx, dim, new, ctxs, (start, prefix))


@pytest.mark.parametrize("new,ctxs,start,prefix", GROUPS[1:3])
@pytest.mark.parametrize("steps", ["one", "up", "down"])
@pytest.mark.parametrize("dim,dtype", [(64, BF), (128, HF)])
def test_scores_as_large_as_fp16_allows(ctx, dim, dtype, steps, new, ctxs, start, prefix):  # noqa: F811
    T.test_scores_as_large_as_fp16_allows(ctx, dim, dtype, steps, new, ctxs, (start, prefix))


@pytest.mark.parametrize("n", [1024, 1025, 1100])
def test_many_groups(ctx, n):  # noqa: F811
    """More groups than the plan keeps in shared memory, some of many rows, some of one member or none."""
    r = random.Random(n)
    start, new, ctxs = [0], [], []
    for g in range(n):
        members = 20 if g % 100 == 7 else 0 if g % 100 == 8 else 1 if g % 100 == 9 else 3
        start.append(start[-1] + members)
        new += [1] * members
        ctxs += [256 + r.randint(0, 20) for _ in range(members)]
    s = Step4(92, new, ctxs, 2, 1, 64, BF, start, [256] * n)
    compare(s, *attend(ctx, s))


@pytest.mark.parametrize("inside,behind", [(1000, 1), (300, 20), (40, 0)])
def test_many_members_inside_the_prefix(ctx, inside, behind):  # noqa: F811
    """Members that end inside the prefix have no keys of their own; a few stand behind it."""
    r = random.Random(inside)
    ctxs = [2048 - r.randint(1, 60) for _ in range(inside)] + [2048 + r.randint(0, 50) for _ in range(behind)]
    s = Step4(93, [1] * len(ctxs), ctxs, 4, 1, 64, BF, [0, len(ctxs)], [2048])
    compare(s, *attend(ctx, s))


@pytest.mark.parametrize("dim,dtype,prefix,members", [(64, BF, 8192, 44), (64, HF, 96, 40), (128, BF, 128, 6)])
def test_a_captured_step_of_groups(dim, dtype, prefix, members):
    """Tables with a shared prefix, append and attention captured as one step, replayed on other lengths: members that end
    inside the prefix, that have no token, that have many."""
    st = torch.cuda.Stream()
    c = rs.Context(W=1, K=1024, stream=st.cuda_stream)
    r = random.Random(prefix)
    heads, kv_heads = 8, 2
    dev = lambda x, t=torch.int32: torch.tensor(x, dtype=t, device="cuda")  # noqa: E731
    n, rows = members + 2, 3 * members + 90
    width = prefix // BLOCK + 12
    blocks = prefix // BLOCK + n * 12 + 5
    cache = empty_cache(rs, blocks, kv_heads, dim)
    ids = r.sample(range(blocks), blocks)
    shared, rest = ids[:prefix // BLOCK], ids[prefix // BLOCK:]
    # the prefix itself
    old = torch.randn(prefix, 2 * kv_heads, dim, generator=torch.Generator().manual_seed(prefix)).to(dtype).cuda()
    rs.kv_append4(c.h, cache, old[:, :kv_heads], old[:, kv_heads:], dev([b * BLOCK + t for b in shared for t in range(BLOCK)], torch.int64))
    table, q_start, kv_len = dev([[-1] * width] * n), dev([0] * (n + 1)), dev([0] * n)
    prev, q_len, free = dev([0] * n), dev([0] * n), dev(rest)
    batch = rs.KVBatch(table, q_start, kv_len, rows, dev([1, 1 + members]), dev([prefix]))   # (one request before the group, one behind)
    pos, slots, counts = dev([0] * rows), dev([0] * rows, torch.int64), dev([0, 0], torch.int64)
    qkv = torch.zeros(rows, heads + 2 * kv_heads, dim, dtype=dtype, device="cuda")
    out, lse = torch.empty(rows, heads, dim, dtype=dtype, device="cuda"), torch.empty(rows, heads, device="cuda")

    def step():
        rs.kv_tables(c.h, batch, q_len, prev, dev_shared, free, pos, slots, counts)
        rs.kv_append4(c.h, cache, qkv[:, heads:heads + kv_heads], qkv[:, heads + kv_heads:], slots)
        rs.kv_attend4(c.h, cache, batch, qkv[:, :heads], dim ** -0.5, out, lse)

    dev_shared = dev([shared])
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        step()
    st.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        step()
    for turn in range(4):
        past = [0] + [prefix] * members + [0]
        new = [5] + [r.choice([1, 1, 1, 2, 0]) for _ in range(members)] + [70 if turn == 2 else 1]
        if turn == 1:     # inside the prefix, of which they write a token each
            past[2], past[3], new[2], new[3] = prefix - 30, 0, 1, 1
        if turn == 3:
            new[4] = 60
        table.fill_(-1)
        for x, y in ((q_len, new), (prev, past)):
            x.copy_(dev(y))
        qkv.copy_(torch.randn(qkv.shape, generator=torch.Generator().manual_seed(turn)).to(dtype))
        out.fill_(7)
        lse.fill_(7)
        torch.cuda.synchronize()
        with torch.cuda.stream(st):
            g.replay()
        st.synchronize()
        s = step_of(cache, table, q_start.tolist(), kv_len.tolist(), qkv[:, :heads], dim ** -0.5)
        assert s.kv_len == [a + b for a, b in zip(past, new)] and s.q_start[-1] == sum(new) <= rows
        compare(s, out, lse)
    rs.kv_status(c.h)
    c.close()


CHILD = r"""
import sys
sys.path[:0] = [sys.argv[1] + "/..", sys.argv[1]]
import pytest
from paper_2606_17081_gb300 import routesim as rs
rs.LIB_PATH = sys.argv[2]
sys.exit(pytest.main(["-x", "-q", "-p", "no:cacheprovider", "-m", "gpu", sys.argv[1] + "/test_gpu_kv4_shared.py", sys.argv[1] + "/test_gpu_kv4_limits.py",
                      sys.argv[1] + "/test_gpu_kv4_lengths.py", sys.argv[1] + "/test_gpu_kv4_attend.py", "-k", sys.argv[3]]))
"""


@pytest.mark.skipif(SHARING, reason="this is the other build")
def test_with_every_prefix_shared(tmp_path):
    B.build()
    obj, lib = str(tmp_path / "kv4_attend_kernel.o"), str(tmp_path / "libroutesim.so")
    src = os.path.join(B.CSRC, "kv4_attend_kernel.cu")
    subprocess.run([B._nvcc(), *B.ARCH, *B.FLAGS, "-DKV4_WORTH=0", "-c", src, "-o", obj], check=True, capture_output=True)
    rest = [os.path.join(B.BUILD, s.replace(".cu", ".o")) for s in B.SOURCES if s != "kv4_attend_kernel.cu"]
    subprocess.run([B._nvcc(), *B.ARCH, "-shared", "-o", lib, obj, *rest, "-lcudart"], check=True, capture_output=True)
    with_groups = "test_gpu_kv4_shared or test_gpu_kv4_limits or test_gpu_kv4_lengths or prefix or members or divide or cut or split or nan or allows or requests_and_groups or beside " \
        "or twice or captured or both_caches or rows or parts"
    r = subprocess.run([sys.executable, "-c", CHILD, HERE, lib, with_groups], capture_output=True, text=True, timeout=600, env={**os.environ, "KV4_SHARES": "1"})
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-2000:]
