"""A kv_attend whose waits run out: the same kernels built with a limit of a few clocks in place of two seconds.  The call ends by itself and writes nothing but its output, the next call reports it
once, and the GPU goes on.  In a process of its own."""
import os
import subprocess
import sys

import pytest

from paper_2606_17081_gb300 import build as B

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CHILD = r"""
import sys
sys.path[:0] = [sys.argv[1], sys.argv[1] + "/tests"]
import torch
from kv_reference import Step
from paper_2606_17081_gb300 import routesim as rs
usual = rs.LIB_PATH
def steps():
    yield Step(0, [1], [700], 8, 2, 128, torch.bfloat16)
    yield Step(1, [1] * 9, [300 + i for i in range(9)], 8, 2, 64, torch.bfloat16, [0, 9], [256])
    yield Step(2, [300, 1, 600], [0, 6000, 2500], 8, 2, 128, torch.bfloat16)   # its loads wait long for free stages
gave_up = []
for lib in (sys.argv[2], usual):
    rs.LIB_PATH, rs._lib = lib, None
    ctx = rs.Context(W=1, K=1024)
    for s in steps():
        cache, batch, q = s.to(rs)
        guard = torch.full((q.shape[0] + 8, *q.shape[1:]), 3.0, dtype=q.dtype, device="cuda")
        out = guard[4:-4]
        report = []
        for call in range(4):
            try:
                rs.kv_attend(ctx.h, cache, batch, q, s.scale, out)
                report.append(0)
            except rs.RoutesimError as e:
                report.append(e.status)
            torch.cuda.synchronize()
        assert (guard[:4] == 3).all() and (guard[-4:] == 3).all()
        # a call that gave up is reported by the next one, which does nothing else
        for a, b in zip(report, report[1:]):
            assert b in (0, rs.RS_ERR_TIMEOUT) and not (a and b), report
        if lib == usual:
            assert not any(report), report
            want, _ = s.expected()
            assert ((out.cpu().double() - want).abs() <= 2.0 ** -5).all()
        else:
            gave_up.append(report == [0, rs.RS_ERR_TIMEOUT, 0, rs.RS_ERR_TIMEOUT])
    ctx.close()
print("GAVE UP", *gave_up)
"""


def built_with(clocks, folder):
    """The library with kv_attend's kernels under another limit."""
    B.build()
    obj, lib = str(folder / "kv_attend_kernel.o"), str(folder / "libroutesim.so")
    src = os.path.join(B.CSRC, "kv_attend_kernel.cu")
    subprocess.run([B._nvcc(), *B.ARCH, *B.FLAGS, f"-DKV_WAIT_CLOCKS={clocks}", "-c", src, "-o", obj], check=True, capture_output=True)
    rest = [os.path.join(B.BUILD, s.replace(".cu", ".o")) for s in B.SOURCES if s != "kv_attend_kernel.cu"]
    subprocess.run([B._nvcc(), *B.ARCH, "-shared", "-o", lib, obj, *rest, "-lcudart"], check=True, capture_output=True)
    return lib


@pytest.mark.parametrize("clocks", [0, 3000])
def test_a_call_that_gives_up_ends_and_is_reported(tmp_path, clocks):
    """0: at the first wait.  3000: somewhere within the runs, or not at all."""
    lib = built_with(clocks, tmp_path)
    r = subprocess.run([sys.executable, "-c", CHILD, ROOT, lib], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    if clocks == 0:
        assert r.stdout.split("GAVE UP")[1].split() == ["True"] * 3, r.stdout


REPLAYED = r"""
import sys
sys.path[:0] = [sys.argv[1], sys.argv[1] + "/tests"]
import torch
from kv_reference import Step
from paper_2606_17081_gb300 import routesim as rs
usual = rs.LIB_PATH
for lib in (sys.argv[2], usual):
    rs.LIB_PATH, rs._lib = lib, None
    st = torch.cuda.Stream()
    ctx = rs.Context(W=1, K=1024, stream=st.cuda_stream)
    rs.kv_status(ctx.h)
    s = Step(0, [1], [700], 8, 2, 128, torch.bfloat16)
    cache, batch, q = s.to(rs)
    out = torch.zeros_like(q)
    torch.cuda.synchronize()
    def status():
        try:
            rs.kv_status(ctx.h)
        except rs.RoutesimError as e:
            return e.status
        return 0
    rs.kv_attend(ctx.h, cache, batch, q, s.scale, out)
    gives_up = rs.RS_ERR_TIMEOUT if lib != usual else 0
    assert [status(), status()] == [gives_up, 0]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=st):
        rs.kv_attend(ctx.h, cache, batch, q, s.scale, out)
        assert status() == rs.RS_ERR_STATE
    assert status() == 0
    with torch.cuda.stream(st):
        g.replay()
        g.replay()
    assert [status(), status()] == [gives_up, 0]
    ctx.close()
print("REPORTED")
"""


def test_a_replay_that_gives_up_is_reported(tmp_path):
    lib = built_with(0, tmp_path)
    r = subprocess.run([sys.executable, "-c", REPLAYED, ROOT, lib], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "REPORTED" in r.stdout, r.stdout + r.stderr
