"""Group norm's statistics where sums of squares lose their digits: equal values
far from 0, rows that say little of the rest of their sample, variances below
FP32's range; and calls larger than a launch."""
import math

import pytest
import torch

from ops_reference import E32

pytestmark = pytest.mark.gpu

# additions that a sum passes at most: 3 in a vector, 64 rows of a thread, 6
# between lanes, 8 between waves
TERMS = 81


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


def run(rt, x, lengths, groups, eps, **how):
    off = torch.tensor([0] + lengths).cumsum(0).int().cuda()
    c = x.shape[1]
    got = rt.group_norm(x.cuda(), torch.ones(c).cuda(), torch.zeros(c).cuda(), groups, offsets=off, eps=eps, **how)
    return [a.cpu().double() for a in got]


def exact(x, lengths, groups, eps):
    parts = x.double().split(lengths)
    v = [p.view(len(p), groups, -1) for p in parts]
    mean = torch.stack([p.mean((0, 2)) for p in v])
    var = torch.stack([((p - m[None, :, None]) ** 2).mean((0, 2)) for p, m in zip(v, mean)])
    return mean, 1 / torch.sqrt(var + eps)


@pytest.mark.parametrize("value", [3.3, 1e5 / 3, 1e10 / 3, -1e20 / 3])
@pytest.mark.parametrize("lengths", [[1, 3, 7, 50], [200, 90, 3], [700, 600], [3000, 5], [2500, 2499]])
def test_equal_values(rt, lengths, value):
    """Variance 0, whatever the value.  Where the FP32 sums are taken, d = mean -
    K has d^2 <= variance + eps, and the sums of d and d^2 are off by TERMS E32
    of themselves: the variance by 3 TERMS E32 (variance + eps), rstd by half of
    that and 8 E32.  The mean is K + d, both known to TERMS E32 of d: a rounding
    of the value and the rounding of d."""
    x = torch.full((sum(lengths), 21), value)
    y, mean, rstd = run(rt, x, lengths, 3, 1e-5)
    want = 1 / math.sqrt(1e-5)
    assert float((rstd - want).abs().max()) <= want * (8 + 1.5 * TERMS) * E32
    # |d| <= TERMS E32 |value|, off by (TERMS + 3) E32 of itself
    v = float(x[0, 0])
    assert float((mean - v).abs().max()) <= abs(v) * E32 * (1 + TERMS * (TERMS + 3) * E32)


@pytest.mark.parametrize("lengths,hint", [([2500], 1), ([2500, 40, 600], 1), ([2500, 40, 600], 0), ([900, 30], 30)])
@pytest.mark.parametrize("cols,groups", [(64, 4), (24, 3), (512, 1)])
def test_rows_that_say_little_of_the_rest(rt, lengths, hint, cols, groups):
    """A sample's first rows are 0, the others lie at 4096 +- 1.  K and the mean
    differ by less than the deviation, or the sums are FP64: the variance is off
    by (terms + 6) E32 (var + d^2) <= 2 (terms + 6) E32 (var + eps) and by the
    mean's own error, 2 d (terms + 3) E32 sqrt(d^2 + var), 3 (terms + 3) E32 (var
    + eps); rstd by half of it and 8 E32.  A thread adds up to 2500 / 8 rows in
    vectors of 4: terms = 330."""
    gen = torch.Generator().manual_seed(1)
    x = torch.randn(sum(lengths), cols, generator=gen) + 4096
    at = 0
    for k in lengths:
        x[at:at + min(8, k // 2)] = 0
        at += k
    y, mean, rstd = run(rt, x, lengths, groups, 1e-5, max_rows=hint)
    mr, rr = exact(x, lengths, groups, 1e-5)
    assert float(((rstd - rr) / rr).abs().max()) <= (8 + 2.5 * 336) * E32
    assert float(((mean - mr) * rr).abs().max()) <= 336 * E32 * 2 + 4096 * E32 * float(rr.max())


@pytest.mark.parametrize("lengths", [[1, 5, 60], [300, 2], [700, 9], [3000, 4]])
@pytest.mark.parametrize("scale", [1e-17, 1e-25, 1e-35])
def test_variances_below_the_range(rt, lengths, scale):
    """eps = 0: FP64 sums, one rounding (and rstd's 8)."""
    gen = torch.Generator().manual_seed(2)
    x = torch.randn(sum(lengths), 16, generator=gen) * scale
    y, mean, rstd = run(rt, x, lengths, 2, 0.0)
    mr, rr = exact(x, lengths, 2, 0.0)
    assert float(((rstd - rr) / rr).abs().max()) <= 8 * E32
    off = (mean - mr) * rr
    assert float(off.abs().max()) <= 8 * E32


def test_more_blocks_than_a_launch_holds(rt):
    """Refused, by either pass, before the workspace is looked at."""
    from paper_2604_15380_amd import PainnError, binding as B
    off = torch.tensor([0, 1 << 16], dtype=torch.int32).cuda()
    some = torch.ones(16).cuda()
    p = some.data_ptr()
    args = dict(precision=1, rows=1 << 16, cols=1 << 20, groups=1 << 15, offsets=off.data_ptr(), n_samples=1, eps=1e-5,
                x=p, ldx=1 << 20, gamma=p, beta=p, y=p, ldy=1 << 20, mean=p, rstd=p)
    with pytest.raises(PainnError, match="blocks") as e:
        B.painn_group_norm(rt.ctx, B.painn_group_norm_args(**args))
    assert e.value.status == -8
    with pytest.raises(PainnError, match="blocks") as e:
        B.painn_group_norm_backward(rt.ctx, B.painn_group_norm_args(**args), p, 1 << 20, p, 1 << 20, p, p)
    assert e.value.status == -8


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["none", "silu", "gelu"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (700, 5), (33, 64)])
def test_sets_of_one_value(rt, dtype, kind, rows, cols):
    """A sample of one row, a column per group: x is its own mean and dx is 0."""
    gen = torch.Generator().manual_seed(3)
    x, dy = (torch.randn(rows, cols, generator=gen).to(dtype).cuda() for _ in range(2))
    g, b = ((1 + torch.randn(cols, generator=gen)).to(dtype).cuda() for _ in range(2))
    how = dict(offsets=torch.arange(rows + 1).int().cuda(), activation=kind)
    y, mean, rstd = rt.group_norm(x, g, b, cols, **how)
    assert torch.equal(mean, x.float())
    if kind == "none":
        assert torch.equal(y, b.expand(rows, cols))
    dx, dg, db = rt.group_norm_backward(dy, x, g, b, mean, rstd, cols, **how)
    assert not bool(dx.any()) and not bool(dg.any())


def test_the_largest_eps(rt):
    """A variance and an eps whose sum leaves FP32: 1 / sqrt(1.4e38 + 3e38)."""
    x = torch.tensor([[1.2e19], [-1.2e19]]).repeat(1, 4)
    y, mean, rstd = run(rt, x, [2], 1, 3e38)
    want = 1 / math.sqrt(float((x.double() ** 2).mean()) + float(torch.tensor(3e38).double()))
    assert float((rstd - want).abs().max()) <= 8 * E32 * want and not bool(mean.any())
