"""Group norm's reverse pass with mean and rstd in other layouts than the
forward's: the same bits as with contiguous ones."""
import pytest
import torch

from test_gpu_group_norm import DTYPES, SHAPES, check_backward, check_forward, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


def turned(a):
    return a.t().contiguous().t()


def apart(a):
    wide = torch.full((2 * a.shape[0], 3 * a.shape[1]), float("nan"), device=a.device)
    return wide[1::2, 2::3].copy_(a)


# short ragged samples, groups of odd widths, equal samples, samples in tiles
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("shape", [5, 6, 8, 13, 15, 17, 18, 21, 22, 23, 24])
def test_any_strides(rt, dtype, shape):
    t, groups = DTYPES[dtype], SHAPES[shape][2]
    data, how, spans = inputs(SHAPES[shape], t, seed=70 + shape)
    x, g, b, dy = (a.cuda() for a in data)
    _, mean, rstd = rt.group_norm(x, g, b, groups, activation="silu", **how)
    want = rt.group_norm_backward(dy, x, g, b, mean, rstd, groups, activation="silu", **how)
    check_backward(data, mean, rstd, spans, groups, "silu", want, t)
    for m, r in ((turned(mean), turned(rstd)), (mean, turned(rstd)), (apart(mean), rstd), (turned(apart(mean)), apart(rstd))):
        got = rt.group_norm_backward(dy, x, g, b, m, r, groups, activation="silu", **how)
        assert all(torch.equal(a, w) for a, w in zip(got, want))


@pytest.mark.parametrize("shape", [5, 15])
def test_shared_values(rt, shape):
    """One mean and rstd that all samples, or all groups, share (stride 0)."""
    groups = SHAPES[shape][2]
    data, how, spans = inputs(SHAPES[shape], torch.float32, seed=90)
    x, g, b, dy = (a.cuda() for a in data)
    gen = torch.Generator().manual_seed(91)
    for m, r in ((torch.randn(1, groups, generator=gen), torch.rand(1, groups, generator=gen) + 0.5),
                 (torch.randn(len(spans), 1, generator=gen), torch.rand(len(spans), 1, generator=gen) + 0.5)):
        m, r = (a.cuda().expand(len(spans), groups) for a in (m, r))
        got = rt.group_norm_backward(dy, x, g, b, m, r, groups, activation="gelu", **how)
        want = rt.group_norm_backward(dy, x, g, b, m.contiguous(), r.contiguous(), groups, activation="gelu", **how)
        assert all(torch.equal(a, w) for a, w in zip(got, want))
        check_backward(data, m, r, spans, groups, "gelu", got, torch.float32)


def test_refusals(rt):
    from paper_2604_15380_amd import PainnError, binding as B
    x, g, stat = torch.ones(6, 12).cuda(), torch.ones(12).cuda(), torch.ones(3, 1).cuda()
    off = torch.tensor([0, 6], dtype=torch.int32).cuda()
    for change in (dict(mean=stat), dict(rstd=stat.double().t()), dict(mean=stat.t().cpu())):
        with pytest.raises(ValueError):
            rt.group_norm_backward(**{**dict(dy=x, x=x, weight=g, bias=g, mean=stat.t(), rstd=stat.t(), groups=3,
                                             offsets=off), **change})
    size = B.painn_group_norm_workspace(1, 6, 12, 3, 1, 0, 0, True)
    space = torch.empty(size, dtype=torch.uint8, device="cuda")
    args = B.painn_group_norm_args(precision=1, rows=6, cols=12, groups=3, offsets=off.data_ptr(), n_samples=1,
                                   x=x.data_ptr(), ldx=12, gamma=g.data_ptr(), beta=g.data_ptr(), mean=stat.data_ptr(),
                                   rstd=stat.data_ptr(), workspace=space.data_ptr(), workspace_bytes=size)
    p = x.data_ptr()
    for strides in ((-3, 1, 3, 1), (3, -1, 3, 1), (3, 1, -1, 1), (3, 1, 3, -1)):
        with pytest.raises(PainnError) as e:
            B.painn_group_norm_backward_strided(rt.ctx, args, strides, p, 12, p, 12, g.data_ptr(), g.data_ptr())
        assert e.value.status == -1


def test_as_many_samples_as_a_call_takes(rt):
    """2^31 - 1 samples, nearly all of them empty, and one in tiles: a row's sample
    is looked up among all of them.  (30 GB)"""
    samples, rows, first = 2**31 - 1, 5000, 10
    offsets = torch.full((samples + 1,), first, dtype=torch.int32, device="cuda")
    offsets[0], offsets[-1] = 0, rows
    gen = torch.Generator().manual_seed(95)
    data = [torch.randn(s, generator=gen) for s in ((rows, 1), (1,), (1,), (rows, 1))]
    x, g, b, dy = (a.cuda() for a in data)
    got = rt.group_norm(x, g, b, 1, offsets=offsets)
    back = rt.group_norm_backward(dy, x, g, b, got[1], got[2], 1, offsets=offsets)
    assert not bool(got[1][1:-1].any()) and not bool(got[2][1:-1].any())
    ends = [0, samples - 1]
    stats = [a[ends] for a in got[1:]]
    spans = [(0, first), (first, rows)]
    check_forward(data, spans, 1, 1e-5, "none", [got[0]] + stats, torch.float32)
    check_backward(data, *stats, spans, 1, "none", back, torch.float32)


def test_no_statistics(rt):
    """Without mean or rstd a call with rows is refused by the library, and one
    without rows does not need them."""
    from paper_2604_15380_amd import PainnError
    x, g, stat = torch.ones(6, 12).cuda(), torch.ones(12).cuda(), torch.ones(1, 3).cuda()
    off = torch.tensor([0, 6], dtype=torch.int32).cuda()
    for m, r in ((None, stat), (stat, None), (None, torch.ones(3, 1).cuda().t()), (None, None)):
        with pytest.raises(PainnError):
            rt.group_norm_backward(x, x, g, g, m, r, 3, offsets=off)
    dx, dw, db = rt.group_norm_backward(x[:0], x[:0], g, g, None, None, 3, offsets=off[:1])
    assert dx.shape == (0, 12) and not bool(dw.any()) and not bool(db.any())
