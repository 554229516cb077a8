"""kv_attend4 on starts and lengths that do not fit together, in steps of every size (bounds: kv4_reference.compare)."""
import pytest

from kv4_reference import Step4, compare
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
