"""The gate over the heads and its reverse pass on the GPU against the plain
64-bit form; indices and counts are equal, bounds in gate_norm_reference."""
import math

import pytest
import torch

import gate_norm_reference as R
from ops_reference import E16, E32, within

pytestmark = pytest.mark.gpu

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
# rows, heads, k
SHAPES = [(1, 1, 1), (1, 16, 2), (200, 16, 2), (7, 3, 3), (1000, 8, 1), (129, 9, 8), (5000, 16, 4), (333, 64, 4),
          (40, 64, 64), (3000, 64, 9), (77, 100, 8), (50, 257, 3), (260, 300, 20), (9, 513, 8), (30, 1024, 5),
          (6, 1000, 1000), (70000, 5, 2), (20000, 64, 2)]


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


def inputs(rows, heads, dtype, seed, masked):
    gen = torch.Generator().manual_seed(seed)
    x = 2 * torch.randn(rows, heads, generator=gen) + torch.randn(heads, generator=gen)
    if masked:
        x[torch.rand(rows, heads, generator=gen) < 0.3] = -math.inf
        x[torch.rand(rows, generator=gen) < 0.1] = -math.inf
    return x.to(dtype), torch.randn(rows, generator=gen), gen


def check_forward(x, k, normalize, got):
    xd = x.double()
    w, idx, counts, share, loss, rows, p = R.gate(xd, k, normalize)
    assert torch.equal(got.indices.cpu(), idx)
    assert torch.equal(got.counts.cpu(), counts)
    assert got.totals.cpu().tolist() == counts.tolist() + [rows]
    e = R.softmax_error(xd)
    within(got.weights.cpu().double() - w, 2 * e * w + 1e-44, "weights")
    # a thread's rows, the lanes, the waves in FP32: rows / 256 + 64 terms at most
    es = (p * e).sum(0) / max(1, rows) + (len(x) / 256 + 64) * E32 * share
    within(got.share.cpu().double() - share, es + 1e-44, "share")
    h, total = x.shape[1], max(1, int(counts.sum()))
    el = h * (counts.double() / total * (es + E32 * share)).sum() + 2 * E32 * loss
    within(got.loss.cpu().double().view(1) - loss, el.view(1) + 1e-44, "loss")
    return idx, counts, rows


def check_backward(x, dw, idx, counts, rows, normalize, balance, got, dtype):
    xd = x.double()
    dx, mag = R.gate_backward(xd, dw.double() if dw is not None else None, idx, counts, rows, normalize, balance)
    # both softmaxes' errors, in the values and in the dot products, and their own sums
    b = (4 * R.softmax_error(xd) + (x.shape[1] + 8) * E32) * mag + 1e-44
    if dtype == torch.bfloat16:
        b = b + E16 * dx.abs()
    within(got.cpu().double() - dx, b, "dlogits")
    assert not bool(got.cpu()[x == -math.inf].any())


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("normalize", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_both_passes(rt, dtype, normalize, shape):
    rows, heads, k = shape
    t = DTYPES[dtype]
    for masked in (False, True):
        x, _, gen = inputs(rows, heads, t, rows + heads, masked)
        g = rt.gate(x.cuda(), k, normalize=normalize)
        idx, counts, n = check_forward(x, k, normalize, g)
        dw = torch.randn(rows, k, generator=gen)
        dw[idx < 0] = math.nan          # places without a head are not used
        got = rt.gate_backward(dw.cuda(), x.cuda(), g, balance=0.3)
        check_backward(x, torch.where(idx < 0, torch.zeros_like(dw), dw), idx, counts, n, normalize, 0.3, got, t)


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_balance_alone(rt, dtype):
    x, _, _ = inputs(700, 16, DTYPES[dtype], 3, True)
    g = rt.gate(x.cuda(), 3)
    idx, counts, n = check_forward(x, 3, False, g)
    got = rt.gate_backward(None, x.cuda(), g, balance=5.0)
    check_backward(x, None, idx, counts, n, False, 5.0, got, DTYPES[dtype])
    assert not bool(rt.gate_backward(None, x.cuda(), g).any())


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("k", [1, 3, 8, 9, 24])
def test_ties_go_to_the_lowest_head(rt, dtype, k):
    """Many equal logits, zeros of both signs among them."""
    gen = torch.Generator().manual_seed(4)
    x = torch.randint(-1, 2, (300, 24), generator=gen).float()
    x[torch.rand(300, 24, generator=gen) < 0.3] = -0.0
    x = x.to(DTYPES[dtype])
    check_forward(x, k, True, rt.gate(x.cuda(), k, normalize=True))


@pytest.mark.parametrize("k", [2, 12])
def test_extreme_logits(rt, k):
    """The type's lowest and largest values are ordinary logits."""
    low, top = torch.finfo(torch.float32).min, torch.finfo(torch.float32).max
    x = torch.zeros(6, 12)
    x[0] = low
    x[1, 3] = top
    x[2] = low
    x[2, 5] = -math.inf
    x[3] = -math.inf
    x[3, 11] = low
    x[4] = torch.linspace(-100, 0, 12)
    g = rt.gate(x.cuda(), k)
    w, idx, counts, share, loss, rows, p = R.gate(x.double(), k, False)
    assert torch.equal(g.indices.cpu(), idx) and torch.equal(g.counts.cpu(), counts)
    assert int(g.totals[-1]) == 6
    assert torch.allclose(g.weights.cpu().double(), w, rtol=3e-5, atol=1e-38)   # 100 E32 in the exponent, 2 spare
    d = rt.gate_backward(torch.ones(6, k).cuda(), x.cuda(), g, balance=1.0)
    assert bool(d.isfinite().all())


@pytest.mark.parametrize("k", [2, 10])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_not_finite_rows(rt, k, dtype):
    x, _, gen = inputs(40, 10, DTYPES[dtype], 5, False)
    y = x.clone()
    y[3, 7], y[9, 2], y[9, 5] = math.nan, math.inf, math.nan
    y[12] = -math.inf
    y[12, 4] = math.nan
    a, b = rt.gate(x.cuda(), k), rt.gate(y.cuda(), k)
    rest = torch.ones(40, dtype=torch.bool)
    rest[[3, 9, 12]] = False
    assert torch.equal(a.weights.cpu()[rest], b.weights.cpu()[rest])
    assert torch.equal(a.indices.cpu()[rest], b.indices.cpu()[rest])
    assert int(b.indices[3, 0]) == 7 and int(b.indices[9, 0]) == 5 and int(b.indices[12, 0]) == 4
    assert bool((b.indices >= -1).all()) and bool((b.indices < 10).all())
    assert bool(b.weights[~rest.cuda()][:, 0].isnan().all()) and bool(b.loss.isnan()) and bool(b.share.isnan().all())
    dw = torch.randn(40, k, generator=gen).cuda()
    d = rt.gate_backward(dw, y.cuda(), b, balance=0.1)
    assert bool(d.cpu()[rest].isfinite().all()) and bool(d.cpu()[3].isnan().all())
    assert not bool(d.cpu()[12][torch.arange(10) != 4].any())


def test_strides_in_place_and_no_rows(rt):
    x, _, gen = inputs(500, 20, torch.float32, 6, True)
    dw = torch.randn(500, 4, generator=gen).cuda()
    want = rt.gate(x.cuda(), 4)
    back = rt.gate_backward(dw, x.cuda(), want, balance=0.2)
    wide = torch.full((500, 27), math.nan, device="cuda")
    wide[:, 2:22] = x.cuda()
    view = wide[:, 2:22]
    got = rt.gate(view, 4)
    for a, b in zip(got[:6], want[:6]):
        assert torch.equal(a, b)
    assert torch.equal(rt.gate_backward(dw, view, got, balance=0.2, dlogits=view), back)
    assert torch.equal(view, back) and bool(wide[:, :2].isnan().all()) and bool(wide[:, 22:].isnan().all())
    empty = rt.gate(x[:0].cuda(), 4)
    assert not bool(empty.counts.any()) and float(empty.loss) == 0 and not bool(empty.share.any())
    assert rt.gate_backward(dw[:0], x[:0].cuda(), empty).shape == (0, 20)


def test_gradient_against_differences(rt):
    """The coefficient 0.7 of the balance loss counts the choices as constants,
    which small moves leave as they are."""
    x, _, gen = inputs(60, 12, torch.float32, 7, True)
    dw = torch.randn(60, 3, generator=gen)
    for normalize in (False, True):
        g = rt.gate(x.cuda(), 3, normalize=normalize)
        dw = torch.where(g.indices.cpu() < 0, torch.zeros_like(dw), dw)
        d = rt.gate_backward(dw.cuda(), x.cuda(), g, balance=0.7).cpu().double()
        u = torch.randn(60, 12, generator=gen, dtype=torch.float64)
        ends = []
        for s in (1e-6, -1e-6):
            w, idx, counts, share, loss, rows, _ = R.gate(x.double() + s * u, 3, normalize)
            assert torch.equal(idx, g.indices.cpu())
            ends.append(float((w * dw).sum() + 0.7 * loss))
        num = (ends[0] - ends[1]) / 2e-6
        assert abs(num - float((d * u).sum())) <= 2e-6 * float((d * u).abs().sum()) + 1e-7


@pytest.mark.parametrize("k", [2, 16])
def test_the_same_bits_every_time_and_in_a_graph(k):
    from paper_2604_15380_amd import Runtime
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        rt = Runtime(0)
        gen = torch.Generator(device="cuda").manual_seed(8)
        x = torch.randn(30001, 16, generator=gen, device="cuda").bfloat16()
        dw = torch.randn(30001, k, generator=gen, device="cuda")
        call = lambda: (lambda g: list(g[:6]) + [rt.gate_backward(dw, x, g, balance=0.1)])(rt.gate(x, k))  # noqa: E731
        want = [a.clone() for a in call()]
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = call()
        for _ in range(3):
            for a in got:
                a.zero_()
            graph.replay()
            eager = call()
            side.synchronize()
            assert all(torch.equal(a, w) and torch.equal(e, w) for a, e, w in zip(got, eager, want))
        del graph
        rt.close()


def test_another_stream(rt):
    x, _, gen = inputs(9000, 16, torch.float32, 9, False)
    x = x.cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        big = torch.randn(4000, 4000, device="cuda")
        big = big @ big
        xs = x + 0 * big[0, 0].nan_to_num(0, 0, 0)
        g = rt.gate(xs, 2)
        d = rt.gate_backward(None, xs, g, balance=1.0) + 0
    side.synchronize()
    idx, counts, n = check_forward(x.cpu(), 2, False, g)
    check_backward(x.cpu(), None, idx, counts, n, False, 1.0, d, torch.float32)


def test_refusals(rt):
    from paper_2604_15380_amd import PainnError, binding as B
    x = torch.randn(300000, 4).cuda()
    g = rt.gate(x, 2)
    for balance in (math.nan, math.inf, 1e39):
        with pytest.raises(PainnError):
            rt.gate_backward(None, x, g, balance=balance)
    with pytest.raises(PainnError, match="1024"):
        rt.gate(torch.zeros(1, 1025).cuda(), 2)
    space = torch.zeros(300 * 6).cuda()
    small = rt.gate(x[:300], 2)
    with pytest.raises(PainnError, match="stride"):
        rt.gate_backward(None, space.as_strided((300, 4), (6, 1)), small, dlogits=space.as_strided((300, 4), (4, 1)))
    args = dict(precision=1, heads=4, rows=300000, k=2, logits=x.data_ptr(), ldx=4, weights=g.weights.data_ptr(),
                indices=g.indices.data_ptr(), counts=g.totals.data_ptr(), share=g.share.data_ptr(), loss=g.loss.data_ptr())
    for change, status in ((dict(), -1), (dict(k=0), -1), (dict(k=5), -1), (dict(rows=-1), -1), (dict(heads=0), -1),
                           (dict(precision=0), -8), (dict(precision=5), -1), (dict(normalize=2), -1), (dict(ldx=3), -1),
                           (dict(logits=None), -1), (dict(rows=1 << 31), -8)):
        with pytest.raises(PainnError) as e:
            B.painn_gate(rt.ctx, B.painn_gate_args(**{**args, **change}))
        assert e.value.status == status, change
