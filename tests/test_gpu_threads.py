"""Contexts of several host threads at once (a context a thread): calls of one kernel that need different amounts of shared
memory must not stand in each other's way."""
import threading
import time

import pytest

from paper_2606_17081_gb300 import routesim as rs

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
