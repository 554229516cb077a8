"""kv_attend on rows that are not finite, or whose scores are as large as the type allows.  Bounds as in
test_gpu_kv_attend."""
import numpy as np
import pytest

from kv_reference import Step
from paper_2606_17081_gb300 import routesim as rs

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

from test_gpu_kv_attend import BF, attend, compare, ctx  # noqa: E402, F401


def past_its_maximum(scale, least, most):
    """A bf16 value x for which 32 x, scaled to powers of two, rounds to something `least` to `most` below itself: the
    largest weight of a row of such scores, taken against the rounded one, is 2^least to 2^most."""
    sl = np.float32(np.float32(scale) * np.float32(1.4426950408889634))
    for k in range(128, 256):
        m = np.float32(32.0 * k * 2.0 ** 22)
        if least <= float(m) * float(sl) - float(np.float32(m * sl)) <= most:
            return k * 2.0 ** 22
    raise AssertionError("no such value")


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,ctxs,groups", [([1], [700], None), ([70], [300], None), ([1] * 6, [260, 300, 256, 290, 400, 257], ([0, 6], [256])),
                                             ([3, 1, 200], [0, 40, 500], None)])
def test_rows_of_nan_beside_rows_of_huge_scores(ctx, dim, new, ctxs, groups):  # noqa: F811
    """Of each kv head's four heads one is NaN, one has finite scores of some 2^35, two are ordinary."""
    s = Step(31, new, ctxs, 8, 2, dim, BF, *(groups or ()))
    x = past_its_maximum(s.scale, 16, 60)
    s.k[..., :32] = torch.where(s.k[..., :32].isnan(), s.k[..., :32], 1.0)
    s.q[..., :32] = 0
    s.q[:, 1::4] = 0
    s.q[:, 1::4, :32] = x
    s.q[:, 2::4] = float("nan")
    out, lse = attend(ctx, s)
    assert out[:, 2::4].isnan().all() and lse[:, 2::4].isnan().all()
    s.q[:, 2::4] = 0
    want, want_lse = s.expected()
    out[:, 2::4], lse[:, 2::4] = want[:, 2::4].to(out), want_lse[:, 2::4].to(lse)
    compare(s, out, lse)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("dtype", [BF, torch.float16])
@pytest.mark.parametrize("steps", ["one", "up", "down"])
@pytest.mark.parametrize("new,ctxs,groups", [([1], [700], None), ([70], [300], None), ([1] * 6, [260, 300, 256, 290, 400, 257], ([0, 6], [256])),
                                             ([3, 1, 200], [0, 40, 500], None)])
def test_scores_as_large_as_fp16_allows(ctx, dim, dtype, steps, new, ctxs, groups):  # noqa: F811
    """Scores of either sign up to 2^35, equal over many keys (every product and sum is exact in 32 bits), beside ordinary
    rows in each kv head's first head."""
    s = Step(32, new, ctxs, 8, 2, dim, dtype, *(groups or ()))
    g = torch.Generator().manual_seed(33)
    longest = max(s.kv_len)
    for i, n in enumerate(s.kv_len):
        for j in range(n):
            at = j / longest
            level = 1.0 if steps == "one" else (1 + int(4 * (at if steps == "up" else 1 - at))) / 8
            s.k[int(s.table[i, j // 16]), :, j % 16, :32] = level * 2.0 ** 15
    s.q[..., :32] = 0
    big = torch.randint(128, 256, (s.rows, 6), generator=g) * (1 - 2 * torch.randint(0, 2, (s.rows, 6), generator=g)) * 2.0 ** 7
    heads = [h for h in range(8) if h % 4]
    s.q[:, heads] = 0
    s.q[:, heads, :32] = big.to(dtype)[:, :, None].expand(-1, -1, 32)
    compare(s, *attend(ctx, s))
