"""Contexts of several host threads at once (a context a thread): calls of one kernel that need different amounts of shared
memory must not stand in each other's way."""
import threading
import time

import numpy as np
import pytest

import oracle as O
from paper_2606_17081_gb300 import routesim as rs
from paper_2606_17081_gb300 import workloads as wk

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)


def together(*calls, seconds=3.0):
    """Each call again and again in a thread of its own; the first error of each."""
    wrong, until = [], time.monotonic() + seconds
    ready = threading.Barrier(len(calls))

    def loop(call):
        ready.wait()
        try:
            while time.monotonic() < until and not wrong:
                call()
        except Exception as e:   # noqa: BLE001
            wrong.append(e)

    threads = [threading.Thread(target=loop, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    if wrong:
        raise wrong[0]


def tables_call(n):
    st = torch.cuda.Stream()
    ctx = rs.Context(W=1, K=1024, stream=st.cuda_stream)
    z = lambda n, t=torch.int32: torch.zeros(n, dtype=t, device="cuda")  # noqa: E731
    b = rs.KVBatch(z((n, 1)), z(n + 1), z(n), n)
    args = (z(n) + 1, z(n), None, torch.arange(n, dtype=torch.int32, device="cuda"), z(n), z(n, torch.int64), z(2, torch.int64))
    torch.cuda.synchronize()
    calls = [0]

    def call():
        rs.kv_tables(ctx.h, b, *args)
        calls[0] += 1
        if calls[0] % 100 == 0:
            st.synchronize()
    return call, lambda: (st.synchronize(), ctx.close(), args[-1].tolist() == [n, n])


def test_block_tables_of_many_and_few_requests():
    many, few = tables_call(16384), tables_call(1)
    together(many[0], few[0])
    assert many[1]()[2] and few[1]()[2]


def route_call(length):
    st = torch.cuda.Stream()
    ctx = rs.Context(W=3, K=4096, n_instances=1, stream=st.cuda_stream)
    n = 4
    tokens = torch.arange(n * length, dtype=torch.int32, device="cuda")
    offsets = torch.arange(n + 1, dtype=torch.int64, device="cuda") * length
    out_len, chosen = torch.ones(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()

    def call():
        rs.route_batch(ctx.h, 0, tokens, offsets, n, out_len, chosen, None, None)
    return call, lambda: (rs.route_active(ctx.h, 0, 3), ctx.close())


def test_routed_prompts_long_and_short():
    long, short = route_call(16 * 1000), route_call(16)
    together(long[0], short[0])
    long[1](), short[1]()


@pytest.mark.parametrize("flags", [0, rs.RS_SIM_TABLES])
def test_simulations_of_long_and_short_prompts(flags):
    """Two threads' replicas, on block ids or hash tables, against the oracle."""
    done = []
    calls = []
    for k, hi in enumerate((200, 16 * 300)):
        tr = wk.make_trace(wk.TraceSpec(n_req=20, len_kind="uniform", len_min=hi // 2, len_max=hi, n_groups=2, prefix_min=16, prefix_max=100,
                                        zipf_s=None, out_kind="uniform", out_min=1, out_max=40), 5 + k)
        rep = wk.Replica(0, 4, wk.POLICY_DYNAMO, 0, 1.0, 0.0, 0, 20)
        st = torch.cuda.Stream()
        ctx = rs.Context(W=3, K=2000, stream=st.cuda_stream)
        want = O.simulate(O.OracleConfig(W=3, K=2000), tr, 4, policy=rep.policy, omega=1.0, tau=0.0, seed=0, n_req=20)["worker"]
        dev = rs.device_trace(tr)
        rec, t = rs.device_records(20, 3)
        torch.cuda.synchronize()

        def call(ctx=ctx, dev=dev, rec=rec, t=t, want=want, rep=rep, st=st):
            res = rs.simulate_replicas(ctx.h, [dev.desc()], rs.RS_MEM_DEVICE, [rs.replica_params(rep)], rec, flags=flags)
            st.synchronize()
            assert res[0].status == rs.RS_OK and np.array_equal(t["worker"].cpu().numpy(), want)
            done.append(1)
        call()
        calls.append(call)
    together(*calls)
    assert len(done) > 4
