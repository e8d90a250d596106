"""Group norm with an activation and its reverse pass on the GPU against the
plain 64-bit form; bounds in gate_norm_reference."""
import math

import pytest
import torch

import gate_norm_reference as R
from ops_reference import ACTS, within

pytestmark = pytest.mark.gpu

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}

# lengths of the samples (None: equal ones, as [samples, rows]), columns, groups
SHAPES = [
    ([1], 1, 1), ([3], 7, 7), ([0, 5, 0, 1, 2, 0], 12, 4), ([96], 337, 1), ([1] * 70, 40, 5),
    ([4, 200, 7, 33, 64, 65, 1, 0, 128], 256, 16), ([20, 9], 254, 2), ([13, 40], 21, 7), ([9, 3], 24, 12),
    ([70, 2], 512, 1), ([5, 6], 1000, 1), ([3, 2], 2048, 1), ([2, 3], 3000, 2), ([300, 11], 48, 48), ([5, 17], 130, 65),
    ([1100, 3, 900], 64, 8), ([5000], 24, 3), ([700, 1, 0, 2500, 13, 1300], 50, 2), ([60] * 130 + [3000] + [5] * 99, 32, 4),
    ([1500], 1100, 1), ([1500], 1100, 2), ((40, 1), 96, 6), ((3, 700), 72, 8), ((2, 2600), 40, 5), ((130, 8), 256, 32), ((5, 64), 128, 1),
]


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


def inputs(shape, dtype, seed=0, tail=0):
    lengths, cols, groups = shape
    gen = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    ragged = isinstance(lengths, list)
    sizes = lengths if ragged else [lengths[1]] * lengths[0]
    rows = sum(sizes) + tail
    ends = [0]
    for k in sizes:
        ends.append(ends[-1] + k)
    level = torch.cat([torch.full((k, 1), v) for k, v in zip(sizes, n(len(sizes)).tolist())] + [torch.zeros(tail, 1)])
    x = n(rows, cols) * torch.exp(0.5 * level) + 2 * level
    t = [a.to(dtype) for a in (x, 1 + 0.2 * n(cols), 0.3 * n(cols), n(rows, cols))]
    how = dict(offsets=torch.tensor(ends, dtype=torch.int32).cuda()) if ragged else dict(sample_rows=lengths[1])
    return t, how, R.sample_spans(ends, rows)


def check_forward(t, spans, groups, eps, kind, got, dtype, **how):
    y, mean, rstd = (a.cpu().double() for a in got)
    x, g, b = (a.double() for a in t[:3])
    yr, mr, rr, xh, z = R.group_norm(x, g, b, groups, spans, eps, kind)
    by, bm, br, _ = R.group_norm_bounds(x, g, b, mr, rr, xh, z, spans, eps, kind, dtype, **how)
    inside = ~yr[:, :1].isnan().expand_as(yr)
    within((y - yr)[inside], by[inside], "y")
    within(mean - mr, bm, "mean")
    within(rstd - rr, br, "rstd")


def check_backward(t, mean, rstd, spans, groups, kind, got, dtype):
    dx, dg, db = (a.cpu().double() if a is not None else None for a in got)
    x, g, b, dy = (a.double() for a in t)
    dxr, dgr, dbr, bx, bg, bb = R.group_norm_backward(dy, x, g, b, mean.cpu().double(), rstd.cpu().double(), groups, spans,
                                                      kind, dtype)
    if dx is not None:
        inside = ~dxr.isnan()
        within((dx - dxr)[inside], bx[inside], "dx")
    within(dg - dgr, bg, "dgamma")
    within(db - dbr, bb, "dbeta")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("k", range(len(SHAPES)))
def test_both_passes(rt, dtype, k):
    t = DTYPES[dtype]
    kind = ACTS[k % 4]
    data, how, spans = inputs(SHAPES[k], t, seed=k)
    groups = SHAPES[k][2]
    x, g, b, dy = (a.cuda() for a in data)
    got = rt.group_norm(x, g, b, groups, activation=kind, **how)
    check_forward(data, spans, groups, 1e-5, kind, got, t)
    back = rt.group_norm_backward(dy, x, g, b, got[1], got[2], groups, activation=kind, **how)
    check_backward(data, got[1], got[2], spans, groups, kind, back, t)


@pytest.mark.parametrize("kind", ACTS)
@pytest.mark.parametrize("shape", [5, 17])
def test_activations(rt, kind, shape):
    data, how, spans = inputs(SHAPES[shape], torch.float32, seed=50)
    groups = SHAPES[shape][2]
    x, g, b, dy = (a.cuda() for a in data)
    got = rt.group_norm(x, g, b, groups, activation=kind, **how)
    check_forward(data, spans, groups, 1e-5, kind, got, torch.float32)
    back = rt.group_norm_backward(dy, x, g, b, got[1], got[2], groups, activation=kind, **how)
    check_backward(data, got[1], got[2], spans, groups, kind, back, torch.float32)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("hint", [0, 1, 40, 5000])
def test_a_hint_changes_no_result(rt, dtype, hint):
    """Also where it is wrong: a sample longer than max_rows."""
    t = DTYPES[dtype]
    data, how, spans = inputs(([700, 1, 0, 2500, 13, 1300], 64, 4), t, seed=3)
    x, g, b, dy = (a.cuda() for a in data)
    got = rt.group_norm(x, g, b, 4, activation="silu", max_rows=hint, **how)
    # (a team of 8 rows at a time then takes 2,500 rows: 313 steps, one row in 40 held)
    check_forward(data, spans, 4, 1e-5, "silu", got, t, terms=330, ratio=40)
    back = rt.group_norm_backward(dy, x, g, b, got[1], got[2], 4, activation="silu", max_rows=hint, **how)
    check_backward(data, got[1], got[2], spans, 4, "silu", back, t)


@pytest.mark.parametrize("lengths", [[4, 9, 0, 30], [900, 3], [6, 1700]])
def test_rows_of_no_sample_stay(rt, lengths):
    data, how, spans = inputs((lengths, 40, 5), torch.float32, seed=4, tail=7)
    first = 3                               # the first sample begins later, too
    off = how["offsets"].clone()
    off[0] = first
    spans = R.sample_spans(off.tolist(), len(data[0]))
    x, g, b, dy = (a.cuda() for a in data)
    # NaN and infinities there reach nothing
    x[:first], x[-7:] = math.inf, math.nan
    dy[:first], dy[-7:] = math.nan, math.inf
    out, dx = torch.full_like(x, 7.5), torch.full_like(x, 7.5)
    got = rt.group_norm(x, g, b, 5, offsets=off, activation="gelu", out=out)
    data[0][:first], data[0][-7:], data[3][:first], data[3][-7:] = 0, 0, 0, 0
    check_forward(data, spans, 5, 1e-5, "gelu", got, torch.float32)
    assert bool((out[:first] == 7.5).all()) and bool((out[-7:] == 7.5).all())
    back = rt.group_norm_backward(dy, x, g, b, got[1], got[2], 5, offsets=off, activation="gelu", dx=dx)
    check_backward(data, got[1], got[2], spans, 5, "gelu", back, torch.float32)
    assert bool((dx[:first] == 7.5).all()) and bool((dx[-7:] == 7.5).all())


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_offsets_outside_the_rows(rt, dtype):
    """Bounds outside [0, rows] are the nearest ones."""
    data, _, _ = inputs(([30, 20], 24, 3), DTYPES[dtype], seed=5)
    off = torch.tensor([-5, 10, 10, 45, 99], dtype=torch.int32)
    spans = R.sample_spans(off.tolist(), 50)
    x, g, b, dy = (a.cuda() for a in data)
    got = rt.group_norm(x, g, b, 3, offsets=off.cuda(), activation="silu")
    check_forward(data, spans, 3, 1e-5, "silu", got, DTYPES[dtype])
    back = rt.group_norm_backward(dy, x, g, b, got[1], got[2], 3, offsets=off.cuda(), activation="silu")
    check_backward(data, got[1], got[2], spans, 3, "silu", back, DTYPES[dtype])


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("shape", [5, 8, 15, 17])
def test_strides_and_in_place(rt, dtype, shape):
    t = DTYPES[dtype]
    data, how, spans = inputs(SHAPES[shape], t, seed=6)
    groups, c = SHAPES[shape][2], SHAPES[shape][1]
    n = len(data[0])
    wide = lambda a: torch.full((n, c + 5), math.nan, dtype=t, device="cuda")[:, 3:3 + c].copy_(a)  # noqa: E731
    x, dy = wide(data[0]), wide(data[3])
    g, b = data[1].cuda(), data[2].cuda()
    want = rt.group_norm(data[0].cuda(), g, b, groups, activation="silu", **how)
    back = rt.group_norm_backward(data[3].cuda(), data[0].cuda(), g, b, want[1], want[2], groups, activation="silu", **how)
    got = rt.group_norm_backward(dy, x, g, b, want[1], want[2], groups, activation="silu", dx=dy, **how)
    assert got[0].data_ptr() == dy.data_ptr()
    assert all(torch.equal(a, w) for a, w in zip(got, back))
    got = rt.group_norm(x, g, b, groups, activation="silu", out=x, **how)
    assert all(torch.equal(a, w) for a, w in zip(got, want))
    base = x._base
    assert bool(base[:, :3].isnan().all()) and bool(base[:, 3 + c:].isnan().all())


def test_far_means_and_ranges(rt):
    """A mean a million times the deviation; squares past FP32's range; values
    so small that eps rules."""
    gen = torch.Generator().manual_seed(8)
    x = torch.randn(60, 32, generator=gen)
    x[:20] = x[:20] + 2.0 ** 20
    x[20:40] *= 1e30
    x[40:] *= 1e-30
    spans = [(0, 20), (20, 40), (40, 60)]
    off = torch.tensor([0, 20, 40, 60], dtype=torch.int32).cuda()
    data = [x, torch.ones(32), torch.zeros(32)]
    got = rt.group_norm(x.cuda(), data[1].cuda(), data[2].cuda(), 4, offsets=off)
    check_forward(data, spans, 4, 1e-5, "none", got, torch.float32)


def test_not_finite_stays_in_its_set(rt):
    data, how, spans = inputs(([40, 3, 1200, 50], 32, 4), torch.float32, seed=9)
    x, g, b, dy = (a.cuda() for a in data)
    clean = rt.group_norm(x, g, b, 4, activation="silu", **how)
    cleanb = rt.group_norm_backward(dy, x, g, b, clean[1], clean[2], 4, activation="silu", **how)
    y = x.clone()
    y[41, 9] = math.nan             # sample 1, group 1
    y[600, 31] = math.inf           # sample 2, group 3
    got = rt.group_norm(y, g, b, 4, activation="silu", **how)
    hit = torch.zeros(len(x), 32, dtype=torch.bool, device="cuda")
    hit[40:43, 8:16] = True
    hit[43:1243, 24:] = True
    assert bool(got[0][hit].isnan().all()) and torch.equal(got[0][~hit], clean[0][~hit])
    back = rt.group_norm_backward(dy, y, g, b, got[1], got[2], 4, activation="silu", **how)
    assert bool(back[0][hit].isnan().all()) and torch.equal(back[0][~hit], cleanb[0][~hit])
    assert bool(back[1][8:16].isnan().all()) and torch.equal(back[1][:8], cleanb[1][:8])


def test_constant_samples(rt):
    """Variance 0: y = act(beta), and with eps = 0 NaN (0 times infinity), as
    the formula says."""
    x = torch.full((30, 16), 3.0).cuda()
    g, b = torch.ones(16).cuda(), torch.linspace(-1, 1, 16).cuda()
    off = torch.tensor([0, 10, 30], dtype=torch.int32).cuda()
    y, mean, rstd = rt.group_norm(x, g, b, 2, offsets=off)
    assert torch.equal(y, b.expand(30, 16)) and bool((mean == 3).all())
    y, mean, rstd = rt.group_norm(x, g, b, 2, offsets=off, eps=0.0)
    assert bool(rstd.isinf().all()) and bool(y.isnan().all())


def test_gradient_against_differences(rt):
    """The FP32 reverse pass along random directions against central differences
    of the 64-bit form."""
    data, how, spans = inputs(([5, 40, 300], 24, 3), torch.float32, seed=10)
    x, g, b, dy = (a.cuda() for a in data)
    _, mean, rstd = rt.group_norm(x, g, b, 3, activation="silu", **how)
    grads = rt.group_norm_backward(dy, x, g, b, mean, rstd, 3, activation="silu", **how)
    gen = torch.Generator().manual_seed(11)
    d64 = [a.double() for a in data]

    def loss(x, g, b):
        return float((R.group_norm(x, g, b, 3, spans, 1e-5, "silu")[0] * d64[3]).sum())

    for i in range(3):
        u = torch.randn(d64[i].shape, generator=gen, dtype=torch.float64)
        h, ends = 1e-5, []
        for s in (h, -h):
            moved = list(d64[:3])
            moved[i] = moved[i] + s * u
            ends.append(loss(*moved))
        num = (ends[0] - ends[1]) / (2 * h)
        ana = grads[i].cpu().double() * u
        assert abs(num - float(ana.sum())) <= 2e-6 * float(ana.abs().sum()) + 1e-7


@pytest.mark.parametrize("rows,cols,groups,samples", [(65502, 256, 16, 1871), (30000, 192, 8, 3), (40000, 64, 64, 40000)])
def test_the_same_bits_every_time(rt, rows, cols, groups, samples):
    gen = torch.Generator(device="cuda").manual_seed(12)
    x = torch.randn(rows, cols, generator=gen, device="cuda").bfloat16()
    dy = torch.randn(rows, cols, generator=gen, device="cuda").bfloat16()
    g = torch.ones(cols, device="cuda", dtype=torch.bfloat16)
    cuts = torch.randperm(rows - 1, generator=torch.Generator().manual_seed(1))[:samples - 1].add(1).sort().values
    off = torch.cat([torch.zeros(1, dtype=torch.int64), cuts, torch.tensor([rows])]).int().cuda()
    first = None
    for _ in range(3):
        y, m, r = rt.group_norm(x, g, g, groups, offsets=off, activation="silu")
        out = (y, m, r) + rt.group_norm_backward(dy, x, g, g, m, r, groups, offsets=off, activation="silu")
        first = first or [a.clone() for a in out]
        assert all(torch.equal(a, f) for a, f in zip(out, first))
    # and against 64 bits at this size, mean and rstd
    ends = off.long()
    xd = x.double().view(rows, groups, -1)
    run = torch.cat([torch.zeros(1, groups, dtype=torch.float64, device="cuda"), xd.sum(2).cumsum(0)])
    n = ((ends[1:] - ends[:-1]) * xd.shape[2]).double()[:, None]
    mean = (run[ends[1:]] - run[ends[:-1]]) / n
    assert float((m - mean).abs().max()) < 1e-6 * float(x.abs().max())


def test_another_stream(rt):
    data, how, spans = inputs(([300, 20, 2000], 64, 8), torch.float32, seed=13)
    x, g, b, dy = (a.cuda() for a in data)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            big = torch.randn(4000, 4000, device="cuda")
            big = big @ big
            xs = x + 0 * big[0, 0].nan_to_num(0, 0, 0)
            got = rt.group_norm(xs, g, b, 8, activation="silu", **how)
            back = rt.group_norm_backward(dy, xs, g, b, got[1], got[2], 8, activation="silu", **how)
            got = [a + 0 for a in got]
            back = [a + 0 for a in back]
    side.synchronize()
    check_forward(data, spans, 8, 1e-5, "silu", got, torch.float32)
    check_backward(data, got[1], got[2], spans, 8, "silu", back, torch.float32)


def test_in_a_graph_beside_another(rt):
    """Two captured graphs of different sizes, replayed in turn with eager work
    between them: each has its own workspace."""
    side = torch.cuda.Stream()
    from paper_2604_15380_amd import Runtime
    with torch.cuda.stream(side):
        mine = Runtime(0)
        sets = []
        for seed, lengths in ((14, [1500, 3, 40]), (15, [9, 2600])):
            data, how, spans = inputs((lengths, 48, 6), torch.bfloat16, seed=seed)
            x, g, b, dy = (a.cuda() for a in data)
            call = lambda x=x, g=g, b=b, dy=dy, how=how: (lambda f: f + mine.group_norm_backward(  # noqa: E731
                dy, x, g, b, f[1], f[2], 6, activation="gelu", **how))(mine.group_norm(x, g, b, 6, activation="gelu", **how))
            want = [a.clone() for a in call()]
            side.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                got = call()
            sets.append((graph, got, want, call))
        for _ in range(3):
            for graph, got, want, call in sets:
                for a in got:
                    a.fill_(math.nan)
                graph.replay()
                sets[0][3]()
                torch.randn(1 << 20, device="cuda").sum()
                side.synchronize()
                assert all(torch.equal(a, w) for a, w in zip(got, want))
        del sets
        mine.close()


def test_no_rows(rt):
    x = torch.empty(0, 12).cuda()
    g = torch.ones(12).cuda()
    off = torch.zeros(4, dtype=torch.int32).cuda()
    y, mean, rstd = rt.group_norm(x, g, g, 3, offsets=off)
    assert y.shape == (0, 12) and not bool(mean.any()) and not bool(rstd.any()) and mean.shape == (3, 3)
    dx, dw, db = rt.group_norm_backward(x, x, g, g, mean, rstd, 3, offsets=off)
    assert not bool(dw.any()) and not bool(db.any())
    # rows, but no samples
    x = torch.ones(5, 12).cuda()
    y, mean, rstd = rt.group_norm(x, g, g, 3, offsets=off[:1], out=torch.full_like(x, 2.0))
    assert mean.shape == (0, 3) and bool((y == 2).all())
    dx, dw, db = rt.group_norm_backward(x, x, g, g, mean, rstd, 3, offsets=off[:1])
    assert not bool(dw.any()) and not bool(db.any())


def test_refusals(rt):
    from paper_2604_15380_amd import PainnError, binding as B
    x, g = torch.ones(6, 12).cuda(), torch.ones(12).cuda()
    off = torch.tensor([0, 6], dtype=torch.int32).cuda()
    for eps in (-1.0, math.nan, math.inf, 1e-60):
        with pytest.raises(PainnError):
            rt.group_norm(x, g, g, 3, offsets=off, eps=eps)
    with pytest.raises(PainnError):
        rt.group_norm(x, g, g, 3, offsets=off, max_rows=-1)
    wide = torch.ones(2, 2049).cuda()
    with pytest.raises(PainnError, match="2048"):
        rt.group_norm(wide, wide[0].clone(), wide[0].clone(), 1, sample_rows=1)
    space = torch.ones(6 * 14).cuda()
    with pytest.raises(PainnError, match="stride"):
        rt.group_norm(space.as_strided((6, 12), (14, 1)), g, g, 3, offsets=off, out=space.as_strided((6, 12), (12, 1)))
    # through the ABI: a workspace that is too small, counts below 0
    big = torch.ones(3000, 12).cuda()
    args = dict(precision=1, activation=0, rows=3000, cols=12, groups=3, offsets=off.data_ptr(), n_samples=1, eps=1e-5,
                x=big.data_ptr(), ldx=12, gamma=g.data_ptr(), beta=g.data_ptr(), y=big.data_ptr(), ldy=12)
    for change, status in ((dict(), -1), (dict(n_samples=-1), -1), (dict(rows=-1), -1), (dict(groups=5), -1),
                           (dict(precision=0), -8), (dict(precision=7), -1), (dict(activation=4), -1), (dict(ldx=11), -1),
                           (dict(reserved=1), -1), (dict(gamma=None), -1), (dict(offsets=None, sample_rows=7), -1),
                           (dict(rows=1 << 31), -8)):
        with pytest.raises(PainnError) as e:
            B.painn_group_norm(rt.ctx, B.painn_group_norm_args(**{**args, **change}))
        assert e.value.status == status, change
