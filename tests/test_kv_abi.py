"""The KV cache operators' C structs and the refusals of the binding, without a GPU."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2606_17081_gb300 import build as B
from paper_2606_17081_gb300 import routesim as rs

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_struct_layout_matches_header(tmp_path):
    structs = {"rs_kv_cache": rs.rs_kv_cache, "rs_kv_batch": rs.rs_kv_batch}
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "routesim.h"', 'int main(void){']
    for sname, cls in structs.items():
        lines.append(f'printf("{sname} %zu\\n", sizeof({sname}));')
        lines += [f'printf("{sname}.{f} %zu\\n", offsetof({sname}, {f}));' for f, _ in cls._fields_]
    lines.append('printf("types %d\\n", RS_BF16 * 10 + RS_FP16); return 0;}')
    src = tmp_path / "probe.c"
    src.write_text("\n".join(lines))
    exe = tmp_path / "probe"
    subprocess.run(["gcc", "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    got = dict(line.split() for line in out.splitlines())
    assert int(got["types"]) == rs.RS_BF16 * 10 + rs.RS_FP16
    for sname, cls in structs.items():
        assert int(got[sname]) == C.sizeof(cls), sname
        for f, _ in cls._fields_:
            assert int(got[f"{sname}.{f}"]) == getattr(cls, f).offset, (sname, f)


def test_entry_points_refuse_a_null_context():
    B.build()
    L = rs.lib()
    cache, batch = rs.rs_kv_cache(), rs.rs_kv_batch()
    assert L.kv_tables(None, C.byref(batch), None, None, None, 0, None, 0, None, None, None) == rs.RS_ERR_INVALID
    assert L.kv_append(None, C.byref(cache), None, None, 0, 0, 0, None) == rs.RS_ERR_INVALID
    assert L.kv_attend(None, C.byref(cache), C.byref(batch), None, 1, 64, 64, 1.0, None, 64, 64, None) == rs.RS_ERR_INVALID
    assert "NULL" in rs.route_last_error(None)


def test_descriptors_refuse_host_tensors():
    k = torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(rs.RoutesimError, match="GPU"):
        rs.KVCache(k, k)
    with pytest.raises(rs.RoutesimError, match="bfloat16 or float16"):
        rs.KVCache(k.float(), k.float())
    i = torch.zeros(1, dtype=torch.int32)
    with pytest.raises(rs.RoutesimError, match="GPU"):
        rs.KVBatch(i[None], i, i, 1)


def test_status_refuses_a_null_context():
    B.build()
    assert rs.lib().kv_status(None) == rs.RS_ERR_INVALID
    with pytest.raises(rs.RoutesimError, match="NULL"):
        rs.kv_status(None)
