"""AdamW over many tensors on the GPU.

The step in FP32 rounds each operation as written, so an elementwise FP32
emulation on the CPU has the same bits, 8-bit codes included; against the
64-bit formula a value is within a few roundings of its terms."""
import math

import pytest
import torch

from ops_reference import E32, within

pytestmark = pytest.mark.gpu

LR, B1, B2, EPS, WD = 6.34e-4, 0.9, 0.999, 1e-8, 0.01
SIZES = [1, 3, 255, 256, 257, 776, 4095, 4096, 4097, 38800, 0, 12345]


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


def encode(x, floor):
    n = x.numel()
    pad = torch.zeros(-(-n // 256) * 256)
    pad[:n] = x
    blocks = pad.view(-1, 256)
    scale = blocks.abs().amax(1) * torch.tensor(1 / 448, dtype=torch.float32)
    scale = torch.where(scale < 2.0 ** -126, torch.zeros_like(scale), scale)
    inv = torch.where(scale == 0, torch.zeros_like(scale), 1.0 / scale)
    q = blocks * inv[:, None]
    if floor:
        q = torch.where(blocks > 0, q.clamp_min(2.0 ** -9), q)
    return q.view(-1)[:n].to(torch.float8_e4m3fn), scale


def decode(code, scale):
    return code.float() * scale.repeat_interleave(256)[:code.numel()]


def step32(p, g, m, v, t, lr=LR, wd=WD):
    """The step with every operation in FP32, on the CPU."""
    m = m * B1 + g * (1 - B1)
    v = v * B2 + (g * g) * (1 - B2)
    root = v.double().sqrt().float()        # torch's own on the CPU is an ulp off at places
    down = torch.tensor(1 / math.sqrt(1 - B2 ** t), dtype=torch.float32)
    p = p * torch.tensor(1 - lr * wd, dtype=torch.float32) - (m * torch.tensor(lr / (1 - B1 ** t), dtype=torch.float32)) / (root * down + torch.tensor(EPS, dtype=torch.float32))
    return p, m, v, root


def make(sizes, seed, spread=True):
    gen = torch.Generator().manual_seed(seed)
    n = lambda k: torch.randn(k, generator=gen)  # noqa: E731
    return [n(k) * 0.05 for k in sizes], [n(k) * 0.01 * (torch.exp(2 * n(k)) if spread else 1.0) for k in sizes]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["fp32", "bf16"])
@pytest.mark.parametrize("copy", [False, True])
def test_steps(rt, bits, grad, copy):
    """Five steps from zero states on tensors of many sizes, one of them empty,
    bit for bit."""
    gt = torch.float32 if grad == "fp32" else torch.bfloat16
    p, _ = make(SIZES, 1)
    dp = [a.cuda() for a in p]
    dg = [torch.zeros(k, dtype=gt, device="cuda") for k in SIZES]
    dc = [torch.zeros(k, dtype=torch.bfloat16, device="cuda") for k in SIZES] if copy else None
    opt = rt.adamw(dp, dg, lr=LR, betas=(B1, B2), eps=EPS, weight_decay=WD, state_bits=bits, copies=dc)
    small = bits == 8
    m = [torch.zeros(k) for k in SIZES]
    v = [torch.zeros(k) for k in SIZES]
    for t in range(1, 6):
        _, g = make(SIZES, 10 + t)
        for d, a in zip(dg, g):
            d.copy_(a)
        opt.step()
        for k in range(len(SIZES)):
            p[k], m[k], v[k], root = step32(p[k], g[k].to(gt).float(), m[k], v[k], t)
            assert torch.equal(dp[k].cpu(), p[k]), (t, SIZES[k])
            if copy:
                assert torch.equal(dc[k].cpu(), p[k].bfloat16())
            if small:
                for a, floor, code, scale in ((m[k], False, opt.m[k], opt.m_scale[k]),
                                              (root, True, opt.v[k], opt.v_scale[k])):
                    rc, rs = encode(a, floor)
                    assert torch.equal(scale.cpu(), rs), (t, SIZES[k])
                    assert torch.equal(code.cpu().view(torch.uint8), rc.view(torch.uint8)), (t, SIZES[k])
                m[k] = decode(*encode(m[k], False))
                r = decode(*encode(root, True))
                v[k] = r * r
            else:
                assert torch.equal(opt.m[k].cpu(), m[k]) and torch.equal(opt.v[k].cpu(), v[k])
    assert opt.steps == 5
    opt.free()


def test_against_64_bits(rt):
    """One step from given FP32 states against the formula in 64 bits."""
    n = 5000
    gen = torch.Generator().manual_seed(4)
    r = lambda: torch.randn(n, generator=gen)  # noqa: E731
    p, g, m, v = 0.05 * r(), 0.01 * r(), 0.01 * r(), (0.01 * r()) ** 2
    d = [a.cuda() for a in (p, g, m.clone(), v.clone())]
    opt = rt.adamw([d[0]], [d[1]], lr=LR, betas=(B1, B2), eps=EPS, weight_decay=WD,
                   state=dict(m=[d[2]], v=[d[3]]), steps=41)
    opt.step(lr=2e-3)
    p, g, m, v = (a.double() for a in (p, g, m, v))
    mr, vr = B1 * m + (1 - B1) * g, B2 * v + (1 - B2) * g * g
    up = 2e-3 * (mr / (1 - B1 ** 42)) / ((vr / (1 - B2 ** 42)).sqrt() + EPS)
    pr = p * (1 - 2e-3 * WD) - up
    mt = 4 * E32 * (m.abs() + g.abs())          # m's terms may cancel
    within(d[2].cpu().double() - mr, mt, "m")
    within(d[3].cpu().double() - vr, 6 * E32 * vr, "v")
    tol = 4 * E32 * p.abs() + up.abs() * 16 * E32 + up.abs() / mr.abs().clamp_min(1e-30) * mt
    within(d[0].cpu().double() - pr, tol, "p")
    assert opt.steps == 42


def test_8_bit_states_hold_what_they_say(rt):
    """Every value of a block is held to 2^-4 of itself or 2^-10 of the
    smallest step; a second moment above zero never becomes zero; zero blocks
    stay zero; an infinity or NaN makes its own block NaN."""
    n = 256 * 5 + 17
    gen = torch.Generator().manual_seed(5)
    g = torch.randn(n, generator=gen) * torch.exp(4 * torch.randn(n, generator=gen))
    g[256:512] = 0
    g[512] = 1e-18
    g[513:768] = 0
    p = torch.zeros(n).cuda()
    dg = g.cuda()
    opt = rt.adamw([p], [dg], lr=1e-3, weight_decay=0.0, state_bits=8)
    opt.step()
    m, r = decode(opt.m[0].cpu(), opt.m_scale[0].cpu()), decode(opt.v[0].cpu(), opt.v_scale[0].cpu())
    mt = g.double() * (1 - 0.9)
    rt_ = g.double().abs() * (1 - 0.999) ** 0.5
    scale_m = opt.m_scale[0].cpu().double().repeat_interleave(256)[:n]
    scale_r = opt.v_scale[0].cpu().double().repeat_interleave(256)[:n]
    big = g.abs() > 1e-17
    assert bool(((m.double() - mt).abs() <= 2.0 ** -4 * mt.abs() * 1.001 + 2.0 ** -10 * scale_m * 1.001)[big].all())
    assert bool(((r.double() - rt_).abs() <= 2.0 ** -4 * rt_ * 1.001 + 2.0 ** -9 * scale_r * 1.001)[big].all())
    assert bool((r[big] > 0).all())
    assert not bool(m[256:512].any()) and not bool(r[256:512].any())
    assert bool(p.isfinite().all())
    dg.zero_()
    dg[0], dg[600] = float("inf"), float("nan")
    opt.step()
    opt.step()
    q = p.cpu()
    assert bool(q[256:512].isfinite().all()) and bool(q[768:].isfinite().all())
    assert bool(q[:256].isnan().all()) and bool(q[512:768].isnan().all())


@pytest.mark.parametrize("bits", [32, 8])
def test_unaligned_tensors(rt, bits):
    """Tensors that start anywhere in an array: the bits of aligned ones, and
    nothing beside them is written."""
    n, shift = 3001, 3
    (p,), (g,) = make([n], 7)
    small = bits == 8
    held = torch.uint8 if small else torch.float32
    pads = {k: torch.full((n + 8,), 5 if t == torch.uint8 else 7.0, dtype=t, device="cuda")
            for k, t in (("p", torch.float32), ("g", torch.bfloat16), ("c", torch.bfloat16), ("m", held), ("v", held))}
    cut = {k: a[shift:shift + n] for k, a in pads.items()}
    cut["p"].copy_(p)
    cut["g"].copy_(g)
    cut["m"].zero_()
    cut["v"].zero_()
    as8 = (lambda a: a.view(torch.float8_e4m3fn)) if small else (lambda a: a)
    st = dict(m=[as8(cut["m"])], v=[as8(cut["v"])])
    if small:
        st.update(m_scale=[torch.zeros(12, device="cuda")], v_scale=[torch.zeros(12, device="cuda")])
    opt = rt.adamw([cut["p"]], [cut["g"]], state_bits=bits, copies=[cut["c"]], state=st)
    q, h = p.cuda(), g.bfloat16().cuda()
    ref = rt.adamw([q], [h], state_bits=bits, copies=[torch.zeros(n, dtype=torch.bfloat16, device="cuda")])
    for _ in range(3):
        opt.step()
        ref.step()
    assert torch.equal(cut["p"], q) and torch.equal(cut["c"], ref.copies[0])
    assert torch.equal(cut["m"], ref.m[0].view(held)) and torch.equal(cut["v"], ref.v[0].view(held))
    for a in pads.values():
        e = 5 if a.dtype == torch.uint8 else 7
        assert bool((a[:shift] == e).all()) and bool((a[shift + n:] == e).all())


def test_resume(rt):
    """A new optimizer from another's states and step count continues it."""
    (p,), (g,) = make([1000], 8)
    a, dg = p.cuda(), g.cuda()
    one = rt.adamw([a], [dg], state_bits=8)
    one.step()
    b = a.clone()
    two = rt.adamw([b], [dg], state_bits=8, steps=one.steps,
                   state={k: [x[0].clone()] for k, x in one.state().items()})
    one.step()
    two.step()
    assert torch.equal(a, b) and one.steps == two.steps == 2


def test_no_tensors(rt):
    opt = rt.adamw([], [])
    opt.step()
    assert opt.steps == 1


def test_refusals(rt):
    from paper_2604_15380_amd import binding as B
    p = torch.zeros(10, device="cuda")
    for call in [lambda: rt.adamw([p], []), lambda: rt.adamw([p], [p.double()]), lambda: rt.adamw([p.double()], [p]),
                 lambda: rt.adamw([p], [p[:9]]), lambda: rt.adamw([p], [p], state_bits=16),
                 lambda: rt.adamw([p.cpu()], [p]), lambda: rt.adamw([p[::2]], [p[:5]]),
                 lambda: rt.adamw([p], [p], copies=[p]), lambda: rt.adamw([p, p], [p, p.bfloat16()])]:
        with pytest.raises(ValueError):
            call()
    for kw in [dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=0.0), dict(weight_decay=-1.0),
               dict(steps=-1), dict(eps=float("nan"))]:
        with pytest.raises(B.PainnError) as e:
            rt.adamw([p], [p.clone()], **kw)
        assert e.value.status == -1
    opt = rt.adamw([p], [p.clone()])
    for lr in (-1.0, float("nan"), float("inf")):
        with pytest.raises(B.PainnError) as e:
            opt.step(lr)
        assert e.value.status == -1
    assert opt.steps == 0
    t = [dict(n=4, param=p.data_ptr(), grad=p.data_ptr(), m=p.data_ptr(), v=None)]
    cfg = dict(beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, state_bits=32, grad_precision=1, steps=0)
    for tt, cc, status in [(t, cfg, -1), ([dict(n=-1)], cfg, -1), ([], {**cfg, "state_bits": 4}, -8),
                           ([], {**cfg, "grad_precision": 0}, -8)]:
        with pytest.raises(B.PainnError) as e:
            B.painn_adamw_create(rt.ctx, tt, cc)
        assert e.value.status == status
