"""Layer norm and its reverse pass on the GPU against the plain 64-bit form.

Bounds, elementwise.  Forward in FP32: the mean is a sum over lanes and
registers, (cols / 64 + 16) roundings of at most the row's largest magnitude
M, and y passes 8 more: (cols / 64 + 24) 2^-24 (M rstd |gamma| + |beta|);
rstd follows the mean's error twice over, which a factor 4 covers.  BF16
adds the output's rounding, 2^-8 |y|.  Reverse: the same with the row's
largest |dy gamma| rstd, times 1 + max |xh| for the projection."""
import pytest
import torch

import ops_reference as ref
from ops_reference import E16, E32, within

pytestmark = pytest.mark.gpu

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
SHAPES = [(1, 1), (3, 7), (1, 256), (96, 337), (130, 64), (5, 511), (9, 1025), (33, 776), (6, 2049), (3, 4099),
          (2, 9001), (5000, 50), (4101, 256)]


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


def inputs(rows, cols, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    x = n(rows, cols) * torch.exp(n(rows, 1)) + n(rows, 1)
    return [t.to(dtype) for t in (x, 1 + 0.2 * n(cols), 0.3 * n(cols), n(rows, cols))]


def forward_bound(x, g, b, y, rs, cols, dtype):
    m = x.abs().amax(1, keepdim=True)
    t = 4 * (cols / 64 + 24) * E32 * (m * rs[:, None] * g.abs() + b.abs())
    return t + (E16 * y.abs() if dtype == torch.bfloat16 else 0)


def check_forward(x, g, b, eps, got, dtype):
    y, mu, rs = got
    xd, gd, bd = x.double(), g.double(), b.double()
    yr, mr, rr = ref.norm(xd, gd, bd, eps)
    cols = x.shape[1]
    within(y.cpu().double() - yr, forward_bound(xd, gd, bd, yr, rr, cols, dtype), "y")
    m = xd.abs().amax(1)
    t = (cols / 64 + 16) * E32 * m
    within(mu.cpu().double() - mr, t, "mean")
    within(rs.cpu().double() - rr, 4 * (cols / 64 + 24) * E32 * rr * (1 + m * rr), "rstd")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_forward(rt, dtype, rows, cols):
    t = DTYPES[dtype]
    x, g, b, _ = inputs(rows, cols, t)
    got = rt.layer_norm(x.cuda(), g.cuda(), b.cuda(), eps=1e-5)
    check_forward(x, g, b, 1e-5, got, t)


def backward_check(rt, x, g, dy, got, mu, rs, dtype):
    dx, dw, db = (None if a is None else a.cpu().double() for a in got)
    xd, gd, dd = x.double(), g.double(), dy.double()
    mu, rs = mu.cpu().double(), rs.cpu().double()
    rx, rw, rb = ref.norm_backward(dd, xd, gd, mu, rs)
    rows, cols = x.shape
    half = E16 if dtype == torch.bfloat16 else 0.0
    xh = ((xd - mu[:, None]) * rs[:, None]).abs()
    # (x - mean) cancels: its rounding is of the size of x
    noise = (xd.abs() + mu.abs()[:, None]) * rs[:, None] * 4 * E32
    if dx is not None:
        a = (dd * gd).abs().amax(1, keepdim=True) * rs[:, None]
        big = xh.amax(1, keepdim=True)
        t = (cols / 64 + 24) * E32 * a * (1 + big) ** 2 + a * (1 + big) * noise.amax(1, keepdim=True) * 2
        within(dx - rx, t + half * rx.abs(), "dx")
    n = rows / 512 + 64
    tw = n * E32 * (dd.abs() * xh).sum(0) + (dd.abs() * noise).sum(0)
    within(dw - rw, tw + half * rw.abs(), "dgamma")
    within(db - rb, n * E32 * dd.abs().sum(0) + half * rb.abs(), "dbeta")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_backward(rt, dtype, rows, cols):
    t = DTYPES[dtype]
    x, g, b, dy = inputs(rows, cols, t, 1)
    _, mu, rs = rt.layer_norm(x.cuda(), g.cuda(), b.cuda())
    got = rt.layer_norm_backward(dy.cuda(), x.cuda(), g.cuda(), mu, rs)
    backward_check(rt, x, g, dy, got, mu, rs, t)
    again = rt.layer_norm_backward(dy.cuda(), x.cuda(), g.cuda(), mu, rs)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("cols", [7, 300])
def test_backward_against_differences(rt, cols):
    """Directional derivatives of a 64-bit forward, by central differences:
    their error is h^2 times the third derivative (1e-8 here) and FP32's."""
    x, g, b, dy = inputs(4, cols, torch.float32, 2)
    _, mu, rs = rt.layer_norm(x.cuda(), g.cuda(), b.cuda())
    dx, dw, db = (t.cpu().double() for t in rt.layer_norm_backward(dy.cuda(), x.cuda(), g.cuda(), mu, rs))
    gen = torch.Generator().manual_seed(3)
    loss = lambda x, g, b: float((ref.norm(x, g, b, 1e-5)[0] * dy.double()).sum())  # noqa: E731
    args = [t.double() for t in (x, g, b)]
    h = 1e-5
    for k, grad in enumerate((dx, dw, db)):
        u = torch.randn(args[k].shape, generator=gen, dtype=torch.float64)
        lo, hi = list(args), list(args)
        lo[k], hi[k] = args[k] - h * u, args[k] + h * u
        num = (loss(*hi) - loss(*lo)) / (2 * h)
        scale = float((grad * u).abs().sum())
        assert abs(num - float((grad * u).sum())) <= 1e-5 * scale


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("cols,ld,shift", [(50, 51, 1), (337, 340, 3), (256, 264, 0), (1500, 1501, 5)])
def test_strides_and_alignment(rt, dtype, cols, ld, shift):
    t = DTYPES[dtype]
    rows = 37
    x, g, b, dy = inputs(rows, cols, t, 4)
    wide = torch.full((rows * ld + shift,), 9.0, dtype=t, device="cuda")

    def view(src=None):
        v = wide.clone()[shift:].view(rows, ld)[:, :cols]
        if src is not None:
            v.copy_(src)
        return v

    out = view()
    got = rt.layer_norm(view(x), g.cuda(), b.cuda(), out=out)
    check_forward(x, g, b, 1e-5, got, t)
    base = out._base if out._base is not None else out
    assert bool((base.view(-1)[:shift] == 9).all()) and bool((base.view(-1)[shift:].view(rows, ld)[:, cols:] == 9).all())
    dx = view()
    res = rt.layer_norm_backward(view(dy), view(x), g.cuda(), got[1], got[2], dx=dx)
    backward_check(rt, x, g, dy, res, got[1], got[2], t)
    assert bool((dx._base.view(-1)[shift:].view(rows, ld)[:, cols:] == 9).all())


def test_in_place(rt):
    x, g, b, dy = inputs(70, 300, torch.float32, 5)
    xc = x.cuda()
    y, mu, rs = rt.layer_norm(xc, g.cuda(), b.cuda(), out=xc)
    assert y.data_ptr() == xc.data_ptr()
    check_forward(x, g, b, 1e-5, (y, mu, rs), torch.float32)
    d = dy.cuda()
    res = rt.layer_norm_backward(d, x.cuda(), g.cuda(), mu, rs, dx=d)
    backward_check(rt, x, g, dy, res, mu, rs, torch.float32)


def test_no_rows(rt):
    e = torch.empty(0, 33, device="cuda")
    g = torch.ones(33, device="cuda")
    y, mu, rs = rt.layer_norm(e, g, g)
    assert y.shape == (0, 33) and mu.shape == (0,)
    dx, dw, db = rt.layer_norm_backward(e, e, g, mu, rs, dweight=g + 1, dbias=g + 2)
    assert dx.shape == (0, 33) and not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_constant_rows_and_nonfinite_values(rt, dtype):
    """A constant row has variance 0: y = beta, rstd = 1 / sqrt(eps).  An
    infinity or NaN stays in its row."""
    t = DTYPES[dtype]
    x, g, b, _ = inputs(12, 100, t, 6)
    x[3] = 2.5
    x[5, 17] = float("inf")
    x[7, 0] = float("nan")
    y, mu, rs = (a.cpu() for a in rt.layer_norm(x.cuda(), g.cuda(), b.cuda(), eps=1e-5))
    assert torch.equal(y[3], b)
    assert abs(float(rs[3]) * 1e-5 ** 0.5 - 1) < 1e-6
    assert bool(y[5].isnan().all()) and bool(y[7].isnan().all())
    rest = [r for r in range(12) if r not in (5, 7)]
    assert bool(y[rest].isfinite().all())


def test_refusals(rt):
    from paper_2604_15380_amd import binding as B
    x, g, b, dy = (t.cuda() for t in inputs(4, 6, torch.float32))
    with pytest.raises(ValueError):
        rt.layer_norm(x.double(), g.double(), b.double())
    with pytest.raises(ValueError):
        rt.layer_norm(x, g[:5], b)
    with pytest.raises(ValueError):
        rt.layer_norm(x.t(), g, b)
    with pytest.raises(ValueError):
        rt.layer_norm(x, g.bfloat16(), b)
    with pytest.raises(ValueError):
        rt.layer_norm(x[:1].expand(4, 6), g, b)
    p = [t.data_ptr() for t in (x, g, b)]
    for prec, rows, cols, ld, eps, ptr, status in [
            (B.PAINN_FP64, 4, 6, 6, 1e-5, p[0], -8), (7, 4, 6, 6, 1e-5, p[0], -1), (1, -1, 6, 6, 1e-5, p[0], -1),
            (1, 4, 0, 6, 1e-5, p[0], -1), (1, 4, 6, 5, 1e-5, p[0], -1), (1, 4, 6, 6, -1.0, p[0], -1),
            (1, 4, 6, 6, float("nan"), p[0], -1), (1, 4, 6, 6, 1e-5, None, -1)]:
        with pytest.raises(B.PainnError) as e:
            B.painn_layer_norm(rt.ctx, prec, rows, cols, ptr, ld, p[1], p[2], eps, p[0], 6, None, None)
        assert e.value.status == status
    with pytest.raises(B.PainnError):      # one of dgamma, dbeta alone
        B.painn_layer_norm_backward(rt.ctx, 1, 4, 6, p[0], 6, p[0], 6, p[1], p[1], p[1], None, 0, p[2], None)
