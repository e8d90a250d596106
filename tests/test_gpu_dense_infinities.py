"""Infinities of both operands in the dense layers and their reverse passes:
what FP32 arithmetic gives.  The 64-bit products on the CPU say which values
are +inf, -inf and NaN (inf - inf, inf times 0); everything else is compared
within the bounds of test_gpu_dense.py."""
import pytest
import torch

from ops_reference import E16, sum_bound

pytestmark = pytest.mark.gpu

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
INF = float("inf")


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


def same(got, a, b, what):
    """got = a b^T with infinities; a [m, k], b [n, k] in 64 bits."""
    want, mag, got = a @ b.t(), a.abs() @ b.t().abs(), got.cpu().double()
    for kind in (torch.isposinf, torch.isneginf, torch.isnan):
        assert torch.equal(kind(got), kind(want)), (what, kind.__name__)
    ok = want.isfinite()
    half = E16 if what.startswith("bf16") else 0.0
    assert bool(((got - want).abs() <= sum_bound(a.shape[1]) * mag + half * want.abs())[ok].all()), what


def operands(n, k, o, dtype, seed):
    """Infinities of either sign in single places, some of both operands at one
    k; a zero opposite an infinity; powers of two, whose lower planes are 0."""
    gen = torch.Generator().manual_seed(seed)
    a, b = (torch.randn(*s, generator=gen).to(dtype).float() for s in ((n, k), (o, k)))
    a[0, k // 2], a[n - 1, k - 1], a[n // 2, 0] = INF, -INF, INF
    b[1, k // 2], b[2, k // 2], b[o - 1, k - 1], b[3, 0] = INF, -INF, INF, 0.0
    b[4], a[1 % n] = 0.5, 2.0
    return a.to(dtype), b.to(dtype)


@pytest.mark.parametrize("dtype", list(DTYPES))
# few rows, tiles of 64, of 128, a width that is no multiple of 8
@pytest.mark.parametrize("n,k,o", [(5, 400, 24), (40, 40, 40), (150, 72, 64), (17000, 64, 256), (33, 57, 19)])
def test_forward(rt, dtype, n, k, o):
    x, w = operands(n, k, o, DTYPES[dtype], n)
    y = rt.linear(x.cuda(), w.cuda())
    same(y, x.double(), w.double(), dtype + " y")
    off = torch.tensor([0, 3, n], dtype=torch.int32, device="cuda")
    y = rt.grouped_linear(x.cuda(), torch.stack([w, -w]).cuda(), off)
    same(y[:3], x[:3].double(), w.double(), dtype + " y, group 0")
    same(y[3:], x[3:].double(), -w.double(), dtype + " y, group 1")


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("n,k,o", [(40, 40, 40), (150, 72, 64), (33, 57, 19)])
def test_backward(rt, dtype, n, k, o):
    # dx[r][i] = sum_o dy[r][o] w[o][i]: contracted over o
    dy, wt = operands(n, o, k, DTYPES[dtype], n + 1)
    w = wt.t().contiguous()
    x = torch.ones(n, k, dtype=DTYPES[dtype])
    dx, _, _ = rt.linear_backward(dy.cuda(), x.cuda(), w.cuda())
    same(dx, dy.double(), wt.double(), dtype + " dx")
    # dw[o][i] = sum_r dy[r][o] x[r][i]: contracted over the rows
    dyt, xt = operands(o, n, k, DTYPES[dtype], n + 2)
    dy, x = dyt.t().contiguous(), xt.t().contiguous()
    _, dw, db = rt.linear_backward(dy.cuda(), x.cuda(), torch.ones(o, k, dtype=DTYPES[dtype], device="cuda"))
    same(dw, dyt.double(), xt.double(), dtype + " dw")
    same(db[:, None], dyt.double(), torch.ones(1, n).double(), dtype + " db")
