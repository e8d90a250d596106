"""The global gradient norm and clipping on the GPU against 64 bits.

Squares are exact in FP64 and n of them leave n 2^-53 of their sum, so the norm
is off by its rounding, E32, and the factor by its own; a product by one more,
E32 or E16."""
import math

import pytest
import torch

from ops_reference import E16, E32, within

pytestmark = pytest.mark.gpu

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
SETS = [[1], [0, 5, 1], [8192], [8191, 8193, 7], [40000] * 3 + [13], [1] * 300, [3_000_001, 2]]


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


def gradients(sizes, dtype, seed=0, scale=1.0):
    """Tensors one behind the other in one array, at any alignment."""
    gen = torch.Generator().manual_seed(seed)
    flat = (torch.randn(sum(sizes) + 1, generator=gen) * scale).to(dtype)[1:].cuda()
    return list(flat.split(sizes))


def norm64(grads):
    return math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))


def check(grads, out, max_norm, norm, factor=None):
    n = norm64(grads)
    total = sum(g.numel() for g in grads)
    assert abs(float(norm) - n) <= (E32 + total * 2.0 ** -53) * n
    f = max_norm / n if n > max_norm else 1.0
    if factor is not None:
        assert abs(float(factor) - f) <= (E32 + total * 2.0 ** -53) * f
    for g, o in zip(grads, out):
        want = g.double() * f
        within(o.double() - want, want.abs() * (2 * E32 + total * 2.0 ** -53 + (E16 if o.dtype == torch.bfloat16 else 0))
               + 1e-44, "clipped")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("k", range(len(SETS)))
@pytest.mark.parametrize("max_norm", [0.5, 1e9])
def test_clip(rt, dtype, k, max_norm):
    t = DTYPES[dtype]
    g = gradients(SETS[k], t, k)
    before = [a.clone() for a in g]
    outs = [torch.full_like(a, math.nan) for a in g]
    c = rt.grad_norm(g, outs=outs)
    norm, factor = c.compute(max_norm)
    check(g, [], max_norm, norm, factor)
    assert float(c.clip(max_norm)) == float(norm)
    check(g, outs, max_norm, norm)
    assert all(torch.equal(a, b) for a, b in zip(g, before))
    c.free()
    c = rt.grad_norm(g)
    assert float(c.clip(max_norm)) == float(norm)
    assert all(torch.equal(a, b) for a, b in zip(g, outs))
    c.free()


def test_mixed_types_and_new_values(rt):
    """The table is of the arrays: their values are read at the call."""
    g = gradients([100, 9000], torch.float32, 1) + gradients([77, 20000], torch.bfloat16, 2)
    c = rt.grad_norm(g)
    for scale in (1.0, 3.0, 1e-3):
        for a in g:
            a.normal_(0, scale)
        before = [a.clone() for a in g]
        norm = c.clip(2.0)
        check(before, g, 2.0, norm)
    c.free()


def test_range(rt):
    """Squares that FP32 cannot hold; a norm beyond FP32 still clips."""
    for v in (1e-30, 1e30, 3e38, 1e-45):
        g = [torch.full((20000,), v).cuda()]
        c = rt.grad_norm(g, outs=[torch.empty_like(g[0])])
        norm, factor = c.compute(1e-3)
        n = norm64(g)
        assert float(norm) == pytest.approx(n, rel=2e-7) if n < 3.4e38 else math.isinf(float(norm))
        c.clip(1e-3)
        if n > 1e-3:
            want = 1e-3 / math.sqrt(20000)
            # (the factor may be below FP32's normal range: 2^-149 apart)
            assert float(c.outs[0][0]) == pytest.approx(want, rel=1e-6 + 2.0 ** -149 * n / 1e-3)
        c.free()


def test_bounds_of_max_norm_and_not_finite(rt):
    g = gradients([5000], torch.float32, 3)
    c = rt.grad_norm(g, outs=[torch.empty_like(g[0])])
    assert float(c.compute()[1]) == 1.0 and float(c.compute(0.0)[1]) == 0.0
    c.clip(0.0)
    assert not bool(c.outs[0].any())
    g[0].zero_()
    norm, factor = c.compute(0.0)
    assert float(norm) == 0.0 and float(factor) == 1.0
    g[0][7] = math.inf
    norm, factor = c.compute(1.0)
    assert math.isinf(float(norm)) and float(factor) == 0.0
    c.clip(1.0)
    assert bool(c.outs[0][7].isnan()) and int(c.outs[0].isnan().sum()) == 1
    g[0][9] = math.nan
    norm, factor = c.compute(1.0)
    assert math.isnan(float(norm)) and math.isnan(float(factor))
    c.clip(1.0)
    assert bool(c.outs[0].isnan().all())
    c.free()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_a_scaled_step_is_a_step_on_scaled_gradients(rt, bits, dtype):
    """In FP32, where the product is the same rounded value in both: the same
    bits.  BF16 gradients are scaled in FP32: as FP32 gradients of those values."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    sizes = [1000, 256, 3, 5000]
    p = [torch.randn(n, generator=gen, device="cuda") for n in sizes]
    g = [torch.randn(n, generator=gen, device="cuda").to(DTYPES[dtype]) for n in sizes]
    q, first = [a.clone() for a in p], [a.clone() for a in p]
    c = rt.grad_norm(g)
    a = rt.adamw(p, g, lr=1e-2, state_bits=bits)
    scaled = [torch.empty(n, device="cuda") for n in sizes]
    b = rt.adamw(q, scaled, lr=1e-2, state_bits=bits)
    for k in range(4):
        for t in g:
            t.normal_(0, 1 + k, generator=gen)
        norm, factor = c.compute(1.5)
        a.step(grad_scale=factor)
        for t, s in zip(g, scaled):
            s.copy_(t.float() * factor)
        b.step()
    assert all(torch.equal(x, y) for x, y in zip(p, q)) and not torch.equal(p[0], first[0])
    sa, sb = a.state(), b.state()
    for k in sa:
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(sa[k], sb[k]))
    for o in (a, b, c):
        o.free()


def test_the_same_bits_every_time_and_in_a_graph():
    from paper_2604_15380_amd import Runtime
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        rt = Runtime(0)
        g = gradients([12_000_000, 40000, 7], torch.bfloat16, 5)
        outs = [torch.empty_like(a) for a in g]
        c = rt.grad_norm(g, outs=outs)
        norm = c.clip(0.5)
        want = [a.clone() for a in outs + [norm]]
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            again = c.clip(0.5)
        for _ in range(3):
            for a in outs:
                a.zero_()
            graph.replay()
            assert all(torch.equal(a, b) for a, b in zip(outs + [again], want))
            for a in outs:
                a.zero_()
            eager = c.clip(0.5)
            assert all(torch.equal(a, b) for a, b in zip(outs + [eager], want))
            side.synchronize()
        del graph
        c.free()
        rt.close()


def test_another_stream(rt):
    side = torch.cuda.Stream()
    g = [torch.zeros(100000, device="cuda")]
    c = rt.grad_norm(g)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        big = torch.randn(4000, 4000, device="cuda")
        big = big @ big
        g[0].copy_(1 + 0 * big[0, 0].nan_to_num(0, 0, 0))
        norm = c.clip(1.0)
        s = g[0].sum()
    side.synchronize()
    assert float(norm) == pytest.approx(math.sqrt(100000), rel=1e-6)
    assert float(s) == pytest.approx(math.sqrt(100000), rel=1e-5)
    c.free()


def test_no_tensors(rt):
    c = rt.grad_norm([])
    norm, factor = c.compute(1.0)
    assert float(norm) == 0.0 and float(factor) == 1.0
    assert float(c.clip(1.0)) == 0.0
    c.free()


def test_a_table_outlives_its_context():
    from paper_2604_15380_amd import PainnError, Runtime
    r = Runtime(0)
    c = r.grad_norm(gradients([10], torch.float32))
    d = r.grad_norm(gradients([10], torch.float32))
    d.free()
    r.close()
    r.ctx = 0
    with pytest.raises(PainnError):
        c.compute(1.0)
    c.free()


def test_refusals(rt):
    from paper_2604_15380_amd import PainnError, binding as B
    a = torch.ones(100).cuda()
    c = rt.grad_norm([a])
    for m in (-1.0, math.nan):
        with pytest.raises(PainnError):
            c.compute(m)
        with pytest.raises(PainnError):
            c.clip(m)
    c.free()
    # the same tensor twice, or overlapping ones, would be scaled twice
    for grads, outs in (([a, a], None), ([a[:60], a[50:]], None), ([a[:50], a[50:]], [a[50:], a[:50]]),
                        ([a[:50]], [a[1:51]])):
        with pytest.raises(PainnError, match="overlaps"):
            rt.grad_norm(grads, outs=outs)
    # ... but may be counted twice where nothing is written
    t = dict(n=100, grad=a.data_ptr(), precision=1)
    h = B.painn_grad_norm_create(rt.ctx, [t, t])
    out = torch.empty(2).cuda()
    B.painn_grad_norm_compute(rt.ctx, h, 1.0, out.data_ptr())
    assert float(out[0]) == pytest.approx(math.sqrt(200), rel=1e-6)
    with pytest.raises(PainnError, match="no place"):
        B.painn_grad_norm_clip(rt.ctx, h, 1.0, out.data_ptr())
    B.painn_grad_norm_free(h)
    for change, status in ((dict(n=-1), -1), (dict(grad=None), -1), (dict(precision=0), -8), (dict(reserved=1), -1),
                           (dict(n=1 << 62), -8)):
        with pytest.raises(PainnError) as e:
            B.painn_grad_norm_create(rt.ctx, [{**t, **change}])
        assert e.value.status == status, change
    with pytest.raises(ValueError):
        rt.grad_norm([a.double()])
    with pytest.raises(ValueError):
        rt.grad_norm([a[::2]])
    with pytest.raises(ValueError):
        rt.grad_norm([a], outs=[a.bfloat16()])
    opt = rt.adamw([a], [torch.ones(100).cuda()])
    with pytest.raises(ValueError):
        opt.step(grad_scale=torch.ones(2).cuda())
    with pytest.raises(ValueError):
        opt.step(grad_scale=torch.ones(1))
    opt.free()
