"""Group norm where a block takes several samples in turn, against 64 bits, and
its optional results.

Whole numbers make the column sums exact: with x and dy of at most 3, means of at
most 1 and rstd of 1 or 2 a product dz xh is at most 24, and sums of 147,456 of
them stay below 2^24, so that in FP32 every order gives the same sum, and a row
that is lost, counted twice or given another sample's statistics shows."""
import pytest
import torch

from ops_reference import E16, E32, within
from test_gpu_group_norm import DTYPES, SHAPES, inputs

pytestmark = pytest.mark.gpu

# rows, columns, groups, samples, equal: waves of a sample each with longer ones,
# many samples of a wave, tiles, blocks of 256 and of 512 threads
SIZES = [(65502, 256, 16, 1871, False), (40000, 64, 64, 40000, False), (60000, 250, 10, 30000, False),
         (30000, 192, 8, 3, False), (120000, 96, 12, 300, True), (147456, 256, 32, 144, True), (90000, 40, 5, 9000, True)]


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


def samples_of(rows, samples, equal):
    """(how group_norm is told, each row's sample, each sample's rows)"""
    if equal:
        ends = torch.arange(samples + 1) * (rows // samples)
    else:
        cuts = torch.randint(0, rows + 1, (samples - 1,), generator=torch.Generator().manual_seed(rows)).sort().values
        ends = torch.cat([torch.zeros(1, dtype=torch.int64), cuts, torch.tensor([rows])])
    count = (ends[1:] - ends[:-1]).cuda()
    ids = torch.arange(samples, device="cuda").repeat_interleave(count)
    return dict(sample_rows=rows // samples) if equal else dict(offsets=ends.int().cuda()), ids, count


def means(a, ids, count):
    """Means over the sets of a [rows, groups, columns], in 64 bits, by row."""
    s = torch.zeros(len(count), a.shape[1], dtype=torch.float64, device="cuda").index_add_(0, ids, a.sum(2))
    return (s / (count.clamp_min(1) * a.shape[2])[:, None])


def spread(stat, ids):
    return stat.double()[ids][:, :, None]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("size", SIZES)
def test_whole_numbers(rt, dtype, size):
    rows, cols, groups, samples, equal = size
    t = DTYPES[dtype]
    how, ids, count = samples_of(rows, samples, equal)
    gen = torch.Generator(device="cuda").manual_seed(cols)
    whole = lambda lo, hi, *s: torch.randint(lo, hi + 1, s, generator=gen, device="cuda").float()  # noqa: E731
    x, dy = whole(-3, 3, rows, cols), whole(-3, 3, rows, cols)
    mean, rstd = whole(-1, 1, samples, groups), whole(1, 2, samples, groups)
    g, b = whole(1, 3, cols), whole(-2, 2, cols)
    for kind in ("none", "relu"):
        dx, dg, db = rt.group_norm_backward(dy.to(t), x.to(t), g.to(t), b.to(t), mean, rstd, groups, activation=kind, **how)
        r = spread(rstd, ids)
        xh = (x.double().view(rows, groups, -1) - spread(mean, ids)) * r
        flat = xh.view(rows, cols)
        dz = dy.double() if kind == "none" else dy.double() * (flat * g + b > 0)
        assert torch.equal(dg, (dz * flat).sum(0).to(t)), kind
        assert torch.equal(db, dz.sum(0).to(t)), kind
        # the means' rounding, their products' and the differences', the last product's
        a = (dz * g).view_as(xh)
        m1, m2 = means(a, ids, count)[ids][:, :, None], means(a * xh, ids, count)[ids][:, :, None]
        want = r * (a - m1 - xh * m2)
        bound = 6 * E32 * r * (a.abs() + m1.abs() + (xh * m2).abs())
        if t == torch.bfloat16:
            bound = bound + E16 * (want.abs() + bound)
        within(dx.double() - want.view(rows, cols), bound.reshape(rows, cols), "dx " + kind)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("size", SIZES)
def test_both_passes(rt, dtype, size):
    """The bounds are gate_norm_reference's; a sample has at most 512 rows where a
    team holds 64 of them, and a column sum passes the rows of a thread, 3 lanes, 8
    waves and the fold's 32 rows and 32 slices (a thread's rows: at most 1 / 1,024
    of all, or the steps of four samples and of two long ones, 150)."""
    rows, cols, groups, samples, equal = size
    t, cg = DTYPES[dtype], cols // groups
    how, ids, count = samples_of(rows, samples, equal)
    gen = torch.Generator(device="cuda").manual_seed(cols + 1)
    n = lambda *s: torch.randn(s, generator=gen, device="cuda")  # noqa: E731
    x = (n(rows, cols) * (0.5 * n(samples, 1)).exp()[ids] + 2 * n(samples, 1)[ids]).to(t)
    g, b, dy = (1 + 0.2 * n(cols)).to(t), (0.3 * n(cols)).to(t), n(rows, cols).to(t)
    y, mean, rstd = rt.group_norm(x, g, b, groups, activation="silu", **how)
    v, gd, bd = x.double().view(rows, groups, cg), g.double(), b.double()
    some = (count > 0).double()[:, None]
    mu = means(v, ids, count)
    var = means((v - spread(mu, ids)) ** 2, ids, count)
    rs = some / torch.sqrt(var + 1e-5)
    top = torch.zeros_like(mu).scatter_reduce_(0, ids[:, None].expand(rows, groups), v.abs().amax(2), "amax")
    terms, ratio = 81, 8
    k = (ratio * var).sqrt() + terms * E32 * top
    d = var.sqrt() + k
    bm = (E32 * mu.abs() + (terms + 3) * E32 * d) * some
    noise = ((terms + 6) * E32 * (var + k ** 2) + 2 * k * (terms + 3) * E32 * d) * rs ** 2 / 2
    br = rs * (8 * E32 + noise)
    within(mean.double() - mu, bm, "mean")
    within(rstd.double() - rs, br, "rstd")
    off = (v - spread(mu, ids)).view(rows, cols)
    row = lambda a: spread(a, ids).expand(rows, groups, cg).reshape(rows, cols)  # noqa: E731
    z = off * row(rs) * gd + bd
    bz = row(rs) * gd.abs() * (row(bm) + 12 * E32 * off.abs()) + E32 * (2 * bd.abs() + z.abs()) + \
        (off * row(rs) * gd).abs() * row(noise + 8 * E32)
    by = 1.13 * bz + 4 * E32 * z.abs()
    want = z * torch.sigmoid(z)
    within(y.double() - want, by + (E16 * (want.abs() + by) if t == torch.bfloat16 else 0), "y")
    # the reverse pass, from the FP32 mean and rstd
    dx, dg, db = rt.group_norm_backward(dy, x, g, b, mean, rstd, groups, activation="silu", **how)
    m, r, dyd = row(mean), row(rstd), dy.double()
    xh = (x.double() - m) * r
    z = xh * gd + bd
    s = torch.sigmoid(z)
    dz = dyd * s * (1 + z * (1 - s))
    exh = 2 * E32 * xh.abs()
    edz = dyd.abs() * (0.8 * (2 * exh * gd.abs() + E32 * z.abs()) + 16 * E32 * (1 + z.abs()))
    a, ea = dz * gd, edz * gd.abs() + E32 * (dz * gd).abs()
    over = lambda q: row(means(q.view(rows, groups, cg), ids, count))  # noqa: E731
    m1, m2 = over(a), over(a * xh)
    em1 = over(ea) + 12 * E32 * over(a.abs())
    em2 = over(ea * xh.abs() + a.abs() * exh) + 14 * E32 * over((a * xh).abs())
    want = r * (a - m1 - xh * m2)
    e = r * (ea + em1 + xh.abs() * em2 + exh * m2.abs() + 6 * E32 * (a.abs() + m1.abs() + (xh * m2).abs()))
    within(dx.double() - want, e * (1 + E16) + E16 * want.abs() if t == torch.bfloat16 else e, "dx")
    k = (max(150, rows / 1024) + 3 + 8 + 64 + 2) * E32
    for got, q, eq, name in ((dg, dz * xh, edz * xh.abs() + dz.abs() * exh, "dgamma"), (db, dz, edz, "dbeta")):
        want, bound = q.sum(0), eq.sum(0) + k * q.abs().sum(0)
        within(got.double() - want, bound + (E16 * want.abs() if t == torch.bfloat16 else 0), name)


# short samples, odd groups, tiles, groups of many columns, equal ones in blocks and in tiles
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("shape", [0, 5, 7, 15, 17, 18, 19, 21, 23, 24])
def test_results_that_are_not_wanted(rt, dtype, shape):
    """Without dx, without dgamma and dbeta, without mean and rstd: the others
    have the same bits."""
    from paper_2604_15380_amd import PainnError, binding as B
    t, (_, cols, groups) = DTYPES[dtype], SHAPES[shape]
    data, how, spans = inputs(SHAPES[shape], t, seed=40 + shape)
    x, g, b, dy = (a.cuda() for a in data)
    y, mean, rstd = rt.group_norm(x, g, b, groups, activation="silu", **how)
    dx, dg, db = rt.group_norm_backward(dy, x, g, b, mean, rstd, groups, activation="silu", **how)
    none, *sums = rt.group_norm_backward(dy, x, g, b, mean, rstd, groups, activation="silu", need_dx=False, **how)
    assert none is None and torch.equal(sums[0], dg) and torch.equal(sums[1], db)
    # through the ABI
    prec = B.PAINN_FP32 if t == torch.float32 else B.PAINN_BF16
    n, each, offsets = len(x), how.get("sample_rows", 0), how.get("offsets")
    spaces = [torch.empty(B.painn_group_norm_workspace(prec, n, cols, groups, len(spans), each, 0, back) + 16,
                          dtype=torch.uint8, device="cuda") for back in (False, True)]
    args = dict(precision=prec, activation=B.ACTIVATIONS["silu"], rows=n, cols=cols, groups=groups,
                offsets=offsets.data_ptr() if each == 0 else None, sample_rows=each, n_samples=len(spans), eps=1e-5,
                x=x.data_ptr(), ldx=cols, gamma=g.data_ptr(), beta=b.data_ptr(), ldy=cols)
    torch.cuda.synchronize()
    out = torch.zeros_like(y)
    B.painn_group_norm(rt.ctx, B.painn_group_norm_args(**args, y=out.data_ptr(), workspace=spaces[0].data_ptr(),
                                                       workspace_bytes=len(spaces[0])))
    back = B.painn_group_norm_args(**args, mean=mean.data_ptr(), rstd=rstd.data_ptr(), workspace=spaces[1].data_ptr(),
                                   workspace_bytes=len(spaces[1]))
    alone = torch.zeros_like(dx)
    call = lambda dw, dbias: B.painn_group_norm_backward(rt.ctx, back, dy.data_ptr(), cols, alone.data_ptr(), cols, dw,  # noqa: E731
                                                         dbias)
    for one in ((dg.data_ptr(), None), (None, db.data_ptr())):
        with pytest.raises(PainnError) as e:
            call(*one)
        assert e.value.status == -1
    call(None, None)
    torch.cuda.synchronize()
    assert torch.equal(out, y) and torch.equal(alone, dx)
