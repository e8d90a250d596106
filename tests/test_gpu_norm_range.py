"""Layer norm's reverse pass on rows whose mean times rstd passes FP32's range:
the places beyond the row, which a row of odd width leaves in the last words,
have no part in it.

x is the same value in every column, so x - mean is exactly 0, rstd is 1 /
sqrt(eps) and dx = rstd (a - mean(a)), a = dy gamma.  The bound: a's rounding
and a sum of c terms, c + 4 roundings of rstd max|a|; BF16 outputs 2^-8."""
import pytest
import torch

from ops_reference import E16, E32, within

pytestmark = pytest.mark.gpu

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


@pytest.mark.parametrize("dtype", list(DTYPES))
# one form of rows each: 16, 32, 64 lanes, two and four words, a whole block, too long to hold
@pytest.mark.parametrize("cols", [17, 70, 141, 300, 700, 1100, 2100, 9001])
@pytest.mark.parametrize("eps", [1e-5, 1e-12])
def test_constant_rows_of_large_values(rt, dtype, cols, eps):
    t = DTYPES[dtype]
    gen = torch.Generator().manual_seed(cols)
    # a power of two: every partial sum of the row and the mean are exact
    size = 2.0 ** (126 - (cols - 1).bit_length())
    x = torch.tensor([size, -size, 1.0])[:, None].repeat(1, cols).to(t)
    dy, g = torch.randn(3, cols, generator=gen).to(t), torch.randn(cols, generator=gen).to(t)
    y, mean, rstd = rt.layer_norm(x.cuda(), g.cuda(), torch.ones(cols, dtype=t, device="cuda"), eps=eps)
    assert torch.equal(mean.cpu(), x[:, 0].float()) and bool((y == 1).all())
    dx, dg, db = rt.layer_norm_backward(dy.cuda(), x.cuda(), g.cuda(), mean, rstd)
    a = dy.double() * g.double()
    want = rstd.cpu().double()[:, None] * (a - a.mean(1, keepdim=True))
    half = E16 if t == torch.bfloat16 else 0.0
    tol = rstd.cpu().double()[:, None] * a.abs().amax(1, keepdim=True) * (cols + 4) * E32 + half * want.abs()
    within(dx.cpu().double() - want, tol, "dx")
    assert not bool(dg.any())
    within(db.cpu().double() - dy.double().sum(0), dy.double().abs().sum(0) * (4 * E32 + half), "db")


@pytest.mark.parametrize("dtype", list(DTYPES))
def test_small_eps(rt, dtype):
    """An eps above 0 that FP32 holds gives constant rows y = beta; one that it
    does not is refused."""
    from paper_2604_15380_amd import PainnError
    t = DTYPES[dtype]
    x, g = torch.full((5, 70), 3.0, dtype=t, device="cuda"), torch.ones(70, dtype=t, device="cuda")
    for eps in (1e-44, 1e-38, 1e-20):
        y, _, rstd = rt.layer_norm(x, g, g, eps=eps)
        assert bool((y == 1).all()) and bool(rstd.isfinite().all()), eps
    for eps in (1e-46, 1e-50, 1e-300):
        with pytest.raises(PainnError) as e:
            rt.layer_norm(x, g, g, eps=eps)
        assert e.value.status == -1
