"""kv_attend4 at the ends of what scales, units and sizes may be.  Bounds as in kv4_reference.compare."""
import math

import pytest

from kv4_reference import Step4, compare
from kv_reference import ref_attend
from paper_2606_17081_gb300 import routesim as rs

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("needs a CUDA device", allow_module_level=True)

from test_gpu_kv4_attend import BF, HF, attend, ctx  # noqa: E402, F401

STEPS = [([1], [700], None), ([1], [9000], None), ([70], [300], None), ([1] * 6, [260, 300, 256, 290, 400, 257], ([0, 6], [256])), ([3, 1, 200], [0, 40, 500], None)]


@pytest.mark.parametrize("new,ctxs,groups", STEPS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q_power,k_power,unit_power", [(-124, -6, 24), (122, 10, -24), (0, 0, 0), (-100, 0, 24), (100, 0, -24), (110, -6, 24)])
def test_scales_that_make_up_for_sizes(ctx, new, ctxs, groups, dim, q_power, k_power, unit_power):  # noqa: F811
    """Ordinary scores of rows and units of extreme sizes: scale * unit alone may be past 2^128 or below 2^-126."""
    s = Step4(81, new, ctxs, 4, 2, dim, BF, *(groups or ()), k_unit=2.0 ** unit_power)
    s.q = (s.q.double() * 2.0 ** q_power).to(BF)
    s.k *= 2.0 ** k_power
    s.scale = 1.23 * dim ** -0.5 * 2.0 ** -(q_power + k_power + unit_power)
    compare(s, *attend(ctx, s))


@pytest.mark.parametrize("new,ctxs,groups", STEPS)
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("unit_power", [0, 24])
def test_the_largest_scale(ctx, new, ctxs, groups, dtype, unit_power):  # noqa: F811
    """Keys of zeros weigh the same; else all weight is on the keys that score highest."""
    s = Step4(82, new, ctxs, 4, 2, 64, dtype, *(groups or ()), k_unit=2.0 ** unit_power)
    empty = s.k.isnan()
    s.k.zero_()
    s.k[:, 1, :, 0] = (torch.arange(s.k.shape[0] * 16).view(-1, 16) * 7 % 23 % 5 + 1) * s.k_unit   # (6 has the code of its own)
    s.k[:, 1, :, 0].clamp_(max=4 * s.k_unit)
    s.k[empty] = float("nan")
    s.q[:, 2:] = 0
    s.q[:, 2:, 0] = 1.0
    s.scale = 3e38
    out, lse = attend(ctx, s)
    s.scale = torch.tensor(s.scale, dtype=torch.float32).item()
    want, want_lse = s.expected()
    far = want_lse.clone()
    far[:, 2:] = torch.where(torch.isinf(far[:, 2:]), far[:, 2:], 0.0)   # (their log sums are past the largest number, and not looked at)
    lse[:, 2:] = far[:, 2:].to(lse)
    s.expected = lambda: (want, far)
    compare(s, out, lse)


@pytest.mark.parametrize("rows_an_sm,more", [(1, 0), (2, 0), (3, -1), (3, 0), (3, 1), (4, 0), (16, 0)])
@pytest.mark.parametrize("dim", [64, 128])
def test_rows_of_parts_around_where_the_join_changes(ctx, rows_an_sm, more, dim):  # noqa: F811
    """Up to three rows an SM have a CTA each to join their parts, more of them a warp: a prompt and single tokens, all cut."""
    heads = 8
    tokens = rows_an_sm * torch.cuda.get_device_properties(0).multi_processor_count // heads + more
    s = Step4(83, [tokens - 2, 1, 1], [3000, 9000, 8000], heads, 2, dim, BF)
    compare(s, *attend(ctx, s))


def check(s, out, lse, step):
    """As kv4_reference.compare, but nothing absolute beside the output's own smallest step: half of it is `step`."""
    want, want_lse = s.expected()
    wide, _ = ref_attend(s.q, s.k, s.v.abs(), s.table.tolist(), s.q_start, s.kv_len, s.scale)
    u = 2.0 ** -8 if s.q.dtype == BF else 2.0 ** -11
    most = s.v[~s.v.isnan()].abs().max().item()
    tol = (2.0 ** -11 * wide + u * want.abs()) * 1.01 + 2.0 ** -14 * wide + 2.0 ** -28 * max(s.kv_len) * most + step
    got, gl = out.cpu().double(), lse.cpu().double()
    assert torch.isfinite(got).all() and ((got - want).abs() <= tol).all()
    assert (want.abs() > 4 * tol).double().mean() > 0.5   # (a wrong factor shows)
    none = torch.isinf(want_lse)
    assert torch.equal(torch.isinf(gl) & (gl < 0), none)
    assert ((gl - want_lse)[~none].abs() <= 2.0 ** -14 + 2.0 ** -20 * want_lse[~none].abs()).all()


@pytest.mark.parametrize("k_power,v_power,dtype", [(9, -24, BF), (9, -24, HF), (-24, -24, BF), (-24, -24, HF), (24, 24, BF), (-20, 13, BF), (-20, 13, HF), (0, -15, HF)])
@pytest.mark.parametrize("new,ctxs,groups", STEPS)
def test_units_to_their_ends(ctx, k_power, v_power, dtype, new, ctxs, groups):  # noqa: F811
    """Results far below one and far above it, held to their own size."""
    size = 600.0 if v_power == -24 else 1.0   # (far above fp16's smallest step, which is 2^-24)
    s = Step4(84, new, ctxs, 4, 2, 64, dtype, *(groups or ()), k_unit=2.0 ** k_power, v_unit=2.0 ** v_power)
    s.v = s.v * size + 1.5 * size * s.v_unit   # (not around 0: long sums stay as large as their terms)
    s.scale /= s.k_unit
    out, lse = attend(ctx, s)
    check(s, out, lse, 2.0 ** -25 if dtype == HF else 0.0)


@pytest.mark.parametrize("power", [17, 20, 24, 26])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("new", [1, 90, 700])
def test_small_weights_alone_make_the_result(ctx, power, dtype, new):  # noqa: F811
    """One key of zeros outweighs each of the others 2^power / 1.3 times: weights are off by 2^-12 of themselves, or by 2^-28 of
    the largest."""
    n = 20000
    s = Step4(85, [new], [n - new], 2, 1, 64, dtype)
    s.k.masked_fill_(~s.k.isnan(), 0.0)
    s.v.masked_fill_(~s.v.isnan(), 1.0)
    at = int(s.table[0, 3])
    s.k[at, :, 5, 0], s.v[at, :, 5] = 6.0, 0.0
    s.q.zero_()
    s.q[:, :, 0] = 8.0
    s.scale = math.log(2.0 ** power / 1.3) / 48.0
    compare(s, *attend(ctx, s))
