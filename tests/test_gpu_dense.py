"""Dense and grouped layers and their reverse passes on the GPU against the
plain 64-bit form.

Bounds, elementwise: a sum of k products is within ops_reference.sum_bound(k)
of the sum of the products' magnitudes; an activation has a slope below 1.13
and is evaluated to 8 roundings of that; BF16 outputs are rounded once (2^-8
of the value at most); where BF16 rounds dz before the products, 2^-8 of the
magnitude sum more."""
import numpy as np
import pytest
import torch

import ops_reference as ref
from ops_reference import ACTS, E16, E32, sum_bound, within

pytestmark = pytest.mark.gpu

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
# rows, d_in, d_out
SHAPES = [(1, 1, 1), (1, 776, 776), (3, 7, 5), (17, 64, 33), (64, 50, 128), (65, 337, 50), (130, 256, 1),
          (200, 33, 257), (129, 130, 129), (700, 776, 130), (2000, 50, 776), (5001, 128, 72)]
GROUPS = [[0, 7], [0, 0, 5, 5, 70], [0, 1, 2, 3, 200, 200, 329], [3, 40, 41, 300],
          list(np.cumsum([0] + [(7 * k) % 13 for k in range(70)])), [0, 2500, 2500, 6000]]


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


def maker(seed, dtype):
    g = torch.Generator().manual_seed(seed)
    return lambda *s, scale=1.0: (torch.randn(*s, generator=g) * scale).to(dtype)


def forward_case(rt, dtype, n, i, o, kind, residual, bias, offsets=None, seed=0):
    t = DTYPES[dtype]
    mk = maker(seed, t)
    G = len(offsets) - 1 if offsets else 1
    x, w, b, r = mk(n, i), mk(G, o, i, scale=i ** -0.5), mk(G, o), mk(n, o)
    ranges = ref.spans(offsets, n) if offsets else [(0, n)]
    d = lambda a: a.double()  # noqa: E731
    yr, zr, mag = ref.linear(d(x), d(w), d(b) if bias else None, kind, d(r) if residual else None, ranges)
    how = dict(activation=kind, residual=r.cuda() if residual else None, keep_preact=True)
    if offsets:
        off = torch.tensor(offsets, dtype=torch.int32).cuda()
        y, z = rt.grouped_linear(x.cuda(), w.cuda(), off, b.cuda() if bias else None, **how)
    else:
        y, z = rt.linear(x.cuda(), w[0].cuda(), b[0].cuda() if bias else None, **how)
    inside = torch.zeros(n, dtype=torch.bool)
    for a, e in ranges:
        inside[a:e] = True
    tz = sum_bound(i) * mag
    ty = 1.13 * tz + 8 * E32 * (yr.abs() + zr.abs() + (r.double().abs() if residual else 0))
    if t == torch.bfloat16:
        tz, ty = tz + E16 * zr.abs(), ty + E16 * yr.abs()
    within((z.cpu().double() - zr)[inside], tz[inside], "z")
    within((y.cpu().double() - yr)[inside], ty[inside], "y")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("n,i,o", SHAPES)
def test_forward(rt, dtype, n, i, o):
    forward_case(rt, dtype, n, i, o, "silu", True, True)
    forward_case(rt, dtype, n, i, o, "none", False, False, seed=1)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("kind", ACTS)
def test_activations(rt, dtype, kind):
    forward_case(rt, dtype, 90, 40, 70, kind, False, True, seed=2)
    backward_case(rt, dtype, 90, 40, 70, kind, kind, seed=2)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("offsets", GROUPS)
def test_grouped_forward(rt, dtype, offsets):
    n = int(max(offsets)) + 4
    forward_case(rt, dtype, n, 50, 72, "silu", False, True, [int(k) for k in offsets])
    forward_case(rt, dtype, n, 129, 33, "gelu", True, True, [int(k) for k in offsets], seed=3)


def backward_case(rt, dtype, n, i, o, kind, x_kind, offsets=None, seed=0):
    t = DTYPES[dtype]
    mk = maker(seed, t)
    G = len(offsets) - 1 if offsets else 1
    dy, z, x, w, xz = mk(n, o), mk(n, o, scale=2.0), mk(n, i), mk(G, o, i, scale=o ** -0.5), mk(n, i, scale=2.0)
    ranges = ref.spans(offsets, n) if offsets else [(0, n)]
    d = lambda a: a.double()  # noqa: E731
    r = ref.linear_backward(d(dy), d(z), kind, d(x), d(w), d(xz), x_kind, ranges)
    how = dict(activation=kind, preact=z.cuda() if kind != "none" else None, x_activation=x_kind,
               x_preact=xz.cuda() if x_kind != "none" else None)
    if offsets:
        off = torch.tensor(offsets, dtype=torch.int32).cuda()
        run = lambda: rt.grouped_linear_backward(dy.cuda(), x.cuda(), w.cuda(), off, **how)  # noqa: E731
    else:
        run = lambda: rt.linear_backward(dy.cuda(), x.cuda(), w[0].cuda(), **how)  # noqa: E731
    got = run()
    dx, dw, db = (a.cpu().double() for a in got)
    if not offsets:
        dw, db = dw[None], db[None]
    inside = torch.zeros(n, dtype=torch.bool)
    for a, e in ranges:
        inside[a:e] = True
    rows = max([e - a for a, e in ranges] + [1])
    half = E16 if t == torch.bfloat16 else 0.0
    dzr = half if kind != "none" else 0.0       # dz is rounded before the products
    rounds = 16 * E32 if kind != "none" or x_kind != "none" else 0.0     # of the slopes
    for name, mine, k in (("dx", dx, o), ("dw", dw, rows), ("db", db, rows)):
        t = (sum_bound(k) + dzr) * r["m" + name] + rounds * r["e" + name] + half * r[name].abs()
        err = mine - r[name]
        within(err[inside] if name == "dx" else err, t[inside] if name == "dx" else t, name)
    again = run()
    keep = inside.cuda()
    assert torch.equal(got[0][keep], again[0][keep])
    assert torch.equal(got[1], again[1]) and torch.equal(got[2], again[2])


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("n,i,o", SHAPES)
def test_backward(rt, dtype, n, i, o):
    backward_case(rt, dtype, n, i, o, "none", "none")
    backward_case(rt, dtype, n, i, o, "silu", "gelu", seed=1)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("offsets", GROUPS)
def test_grouped_backward(rt, dtype, offsets):
    n = int(max(offsets)) + 4
    backward_case(rt, dtype, n, 50, 72, "silu", "none", [int(k) for k in offsets])
    backward_case(rt, dtype, n, 129, 33, "none", "silu", [int(k) for k in offsets], seed=3)


@pytest.mark.parametrize("grouped", [False, True])
def test_backward_against_differences(rt, grouped):
    """Directional derivatives of the 64-bit layer by central differences; the
    gradients come from FP32 outputs of the forward (z to 2^-24)."""
    n, i, o, G = 23, 19, 21, 3
    mk = maker(9, torch.float32)
    x, w, b, dy = mk(n, i), mk(G, o, i, scale=i ** -0.5), mk(G, o), mk(n, o)
    offsets = [0, 9, 9, 23]
    ranges = ref.spans(offsets, n) if grouped else [(0, n)]
    if grouped:
        off = torch.tensor(offsets, dtype=torch.int32).cuda()
        _, z = rt.grouped_linear(x.cuda(), w.cuda(), off, b.cuda(), activation="gelu", keep_preact=True)
        g = rt.grouped_linear_backward(dy.cuda(), x.cuda(), w.cuda(), off, activation="gelu", preact=z)
    else:
        w, b = w[:1], b[:1]
        _, z = rt.linear(x.cuda(), w[0].cuda(), b[0].cuda(), activation="gelu", keep_preact=True)
        g = rt.linear_backward(dy.cuda(), x.cuda(), w[0].cuda(), activation="gelu", preact=z)
    grads = [g[0].cpu().double(), g[1].cpu().double().view(w.shape), g[2].cpu().double().view(b.shape)]
    args = [t.double() for t in (x, w, b)]
    loss = lambda x, w, b: float((ref.linear(x, w, b, "gelu", None, ranges)[0] * dy.double()).sum())  # noqa: E731
    gen = torch.Generator().manual_seed(1)
    for k in range(3):
        u = torch.randn(args[k].shape, generator=gen, dtype=torch.float64)
        lo, hi = list(args), list(args)
        lo[k], hi[k] = args[k] - 1e-5 * u, args[k] + 1e-5 * u
        num = (loss(*hi) - loss(*lo)) / 2e-5
        scale = float((grads[k] * u).abs().sum())
        assert abs(num - float((grads[k] * u).sum())) <= 1e-5 * scale


def strided(src, ld, shift):
    rows, cols = src.shape
    base = torch.full((rows * ld + shift,), 7.0, dtype=src.dtype, device="cuda")
    v = base[shift:].view(rows, ld)[:, :cols]
    v.copy_(src)
    return v


def untouched(v, ld, shift):
    base = v._base.view(-1)
    rest = base[shift:].view(-1, ld)[:, v.shape[1]:]
    return bool((base[:shift] == 7).all()) and bool((rest == 7).all())


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("i,o,extra,shift", [(48, 40, 8, 0), (48, 40, 1, 1), (51, 37, 3, 5), (200, 136, 5, 7)])
def test_strides_and_alignment(rt, dtype, i, o, extra, shift):
    """Row strides above the width and bases that are not 16-byte aligned, in
    every operand; bits are those of contiguous operands, and what lies
    between the rows is left alone."""
    n = 150
    mk = maker(5, DTYPES[dtype])
    x, w, b, r, dy, xz = mk(n, i), mk(o, i), mk(o), mk(n, o), mk(n, o), mk(n, i)
    y0, z0 = rt.linear(x.cuda(), w.cuda(), b.cuda(), activation="silu", residual=r.cuda(), keep_preact=True)
    y = strided(torch.zeros(n, o, dtype=x.dtype), o + extra, shift)
    sx, sr = strided(x, i + extra, shift), strided(r, o + extra, shift)
    y1, z1 = rt.linear(sx, w.cuda(), b.cuda(), activation="silu", residual=sr, keep_preact=True, out=y)
    assert torch.equal(y0, y1) and torch.equal(z0, z1) and untouched(y, o + extra, shift)
    rt.linear(sx, w.cuda(), b.cuda(), activation="silu", residual=sr, out=sr)      # in place of the residual
    assert torch.equal(sr, y0)
    how = dict(activation="silu", x_activation="silu")
    a = rt.linear_backward(dy.cuda(), x.cuda(), w.cuda(), preact=z0, x_preact=xz.cuda(), **how)
    dx = strided(torch.zeros(n, i, dtype=x.dtype), i + extra, shift)
    c = rt.linear_backward(strided(dy, o + extra, shift), sx, w.cuda(), preact=strided(z0, o + extra, shift),
                           x_preact=strided(xz, i + extra, shift), dx=dx, **how)
    assert all(torch.equal(p, q) for p, q in zip(a, c)) and untouched(dx, i + extra, shift)


def test_rows_outside_the_groups(rt):
    """Rows of no group keep what they hold; bounds past the rows end there."""
    mk = maker(6, torch.float32)
    x, w = mk(100, 30).cuda(), mk(2, 20, 30).cuda()
    out = torch.full((100, 20), 5.0, device="cuda")
    off = torch.tensor([10, 40, 400], dtype=torch.int32).cuda()
    rt.grouped_linear(x, w, off, out=out)
    assert bool((out[:10] == 5).all()) and bool((out[10:] != 5).all())
    off = torch.tensor([10, 40, 60], dtype=torch.int32).cuda()
    out.fill_(5.0)
    rt.grouped_linear(x, w, off, out=out)
    assert bool((out[60:] == 5).all()) and bool((out[:10] == 5).all())
    dx = torch.full((100, 30), 5.0, device="cuda")
    rt.grouped_linear_backward(mk(100, 20).cuda(), x, w, off, dx=dx)
    assert bool((dx[60:] == 5).all()) and bool((dx[:10] == 5).all()) and bool((dx[10:60] != 5).all())


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_no_rows(rt, dtype):
    t = DTYPES[dtype]
    e_in, e_out = torch.empty(0, 9, dtype=t, device="cuda"), torch.empty(0, 11, dtype=t, device="cuda")
    w = torch.ones(3, 11, 9, dtype=t, device="cuda")
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    assert rt.linear(e_in, w[0]).shape == (0, 11)
    assert rt.grouped_linear(e_in, w, off).shape == (0, 11)
    for got in (rt.linear_backward(e_out, e_in, w[0], dweight=w[0] + 1),
                rt.grouped_linear_backward(e_out, e_in, w, off, dweight=w + 1)):
        assert got[0].shape == (0, 9) and not got[1].any() and not got[2].any()


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_nonfinite_values(rt, dtype):
    """An infinity or NaN of x reaches its own row only, as in FP32 arithmetic:
    inf times a weight above zero is inf."""
    t = DTYPES[dtype]
    mk = maker(7, t)
    x, w = mk(140, 100), mk(60, 100).abs() + 0.5
    x[3, 5], x[70, 99], x[139, 0] = float("inf"), float("nan"), float("-inf")
    y = rt.linear(x.cuda(), w.cuda()).cpu()
    assert bool((y[3] == float("inf")).all()) and bool(y[70].isnan().all()) and bool((y[139] == -float("inf")).all())
    rest = [k for k in range(140) if k not in (3, 70, 139)]
    assert bool(y[rest].isfinite().all())


def test_fp32_range(rt):
    """FP32 operands near the ends of their range."""
    x = torch.tensor([[3.0e38, 1.0], [1e-30, 2e-36], [-3.3e38, 0.0]]).cuda()
    w = torch.tensor([[0.5, 1.0], [1.0, 1e-3]]).cuda()
    y = rt.linear(x, w).cpu().double()
    r = x.cpu().double() @ w.cpu().double().t()
    assert bool(((y - r).abs() <= 4e-7 * r.abs()).all())


def test_refusals(rt):
    from paper_2604_15380_amd import binding as B
    mk = maker(8, torch.float32)
    x, w, b, dy = mk(6, 5).cuda(), mk(4, 5).cuda(), mk(4).cuda(), mk(6, 4).cuda()
    off = torch.tensor([0, 6], dtype=torch.int32).cuda()
    bad = [lambda: rt.linear(x.double(), w.double()), lambda: rt.linear(x, w.bfloat16()), lambda: rt.linear(x, w.t()),
           lambda: rt.linear(x, w, b[:3]), lambda: rt.linear(x, w, b, activation="tanh"),
           lambda: rt.linear(x.t(), w), lambda: rt.linear(x, w, residual=x), lambda: rt.linear(x[:1].expand(6, 5), w),
           lambda: rt.linear(x.cpu(), w), lambda: rt.linear(x, w, out=dy[:5]),
           lambda: rt.grouped_linear(x, w, off), lambda: rt.grouped_linear(x, w[None], off.long()),
           lambda: rt.grouped_linear(x, w[None], off[:1]), lambda: rt.grouped_linear(x, w[None], None),
           lambda: rt.linear_backward(dy, x, w, activation="silu"),
           lambda: rt.linear_backward(dy, x, w, x_activation="silu"),
           lambda: rt.linear_backward(dy[:, :3], x, w)]
    for call in bad:
        with pytest.raises(ValueError):
            call()

    def args(**kw):
        a = dict(precision=1, activation=0, rows=6, d_in=5, d_out=4, x=x.data_ptr(), ldx=5, w=w.data_ptr(),
                 y=dy.data_ptr(), ldy=4)
        a.update(kw)
        return B.painn_linear_args(**a)

    for kw, status in [(dict(precision=0), -8), (dict(precision=3), -1), (dict(activation=9), -1), (dict(rows=-1), -1),
                       (dict(d_in=0), -1), (dict(d_out=1 << 21, ldy=1 << 21), -8), (dict(x=None), -1),
                       (dict(ldx=4), -1), (dict(ldy=3), -1), (dict(z=x.data_ptr(), ldz=2), -1),
                       (dict(rows=1 << 62, ldx=5), -8)]:
        with pytest.raises(B.PainnError) as e:
            B.painn_linear(rt.ctx, args(**kw))
        assert e.value.status == status, kw
    for n, o, status in [(0, off.data_ptr(), -1), (5000, off.data_ptr(), -1), (1, None, -1)]:
        with pytest.raises(B.PainnError) as e:
            B.painn_grouped_linear(rt.ctx, args(), n, o)
        assert e.value.status == status
    back = dict(precision=1, activation=0, rows=6, d_in=5, d_out=4, dy=dy.data_ptr(), lddy=4, x=x.data_ptr(), ldx=5,
                w=w.data_ptr())
    for kw in [dict(dbias=b.data_ptr()), dict(dy=None, dx=x.data_ptr(), lddx=5), dict(dx=x.data_ptr(), lddx=4),
               dict(activation=1, dx=x.data_ptr(), lddx=5), dict(x_activation=1, dx=x.data_ptr(), lddx=5)]:
        with pytest.raises(B.PainnError) as e:
            B.painn_linear_backward(rt.ctx, B.painn_linear_backward_args(**{**back, **kw}))
        assert e.value.status == -1, kw


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("i", [127, 128, 129, 136, 255, 256, 257, 264, 1030])
def test_few_rows_of_any_inner_length(rt, dtype, i):
    forward_case(rt, dtype, 19, i, 45, "silu", True, True, seed=i)
    forward_case(rt, dtype, 33, i, 40, "gelu", True, True, [0, 0, 1, 18, 18, 33], seed=i + 1)


@pytest.mark.parametrize("n,i,o,offsets", [(28, 257, 1, None), (5, 64, 1, None), (1, 776, 776, None),
                                           (40, 130, 200, None), (8192, 40, 1, None), (128, 72, 64, [0, 1, 1, 90, 126]),
                                           (129, 45, 37, [0, 2, 60, 60, 129])])
def test_few_values_of_dz_are_not_rounded(rt, n, i, o, offsets):
    # dz as a BF16 value and a BF16 remainder is 2^-16 off, E16 squared
    t, mk = torch.bfloat16, maker(n + i, torch.bfloat16)
    G = len(offsets) - 1 if offsets else 1
    dy, z, x, w = mk(n, o), mk(n, o, scale=2.0), mk(n, i), mk(G, o, i, scale=o ** -0.5)
    ranges = ref.spans(offsets, n) if offsets else [(0, n)]
    r = ref.linear_backward(dy.double(), z.double(), "silu", x.double(), w.double(), None, "none", ranges)
    how = dict(activation="silu", preact=z.cuda())
    if offsets:
        got = rt.grouped_linear_backward(dy.cuda(), x.cuda(), w.cuda(), torch.tensor(offsets, dtype=torch.int32).cuda(), **how)
    else:
        got = rt.linear_backward(dy.cuda(), x.cuda(), w[0].cuda(), **how)
    inside = torch.zeros(n, dtype=torch.bool)
    for a, e in ranges:
        inside[a:e] = True
    rows = max([e - a for a, e in ranges] + [1])
    for name, mine, k in (("dx", got[0], o), ("dw", got[1], rows)):
        mine = mine.cpu().double().reshape(r[name].shape)
        tol = (sum_bound(2 * k) + E16 * E16) * r["m" + name] + 16 * E32 * r["e" + name] + E16 * r[name].abs()
        err = mine - r[name]
        within(err[inside] if name == "dx" else err, tol[inside] if name == "dx" else tol, name)


def test_infinite_gradients_stay_infinite(rt):
    dy = torch.ones(3, 8, dtype=torch.bfloat16)
    dy[1, 2] = float("inf")
    z, x, w = torch.full((3, 8), 2.0), torch.ones(3, 16), torch.ones(8, 16)
    z, x, w = (a.to(torch.bfloat16).cuda() for a in (z, x, w))
    dx, dw, db = rt.linear_backward(dy.cuda(), x, w, activation="silu", preact=z)
    assert torch.isinf(dx[1]).all() and torch.isfinite(dx[0]).all() and torch.isfinite(dx[2]).all()
    assert torch.isinf(dw[2]).all() and torch.isfinite(dw[:2]).all() and torch.isinf(db[2])
