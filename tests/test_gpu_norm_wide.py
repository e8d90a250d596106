"""Layer norm on rows of millions of columns, where the columns' sums take
several rounds of a launch; rows longer than its counters hold are refused.

Bounds as a sum of c terms by 256 threads has them: (c / 256 + 16) roundings
of the sum of the magnitudes for the row's sums; the column sums over two rows
are two roundings of theirs.  BF16 outputs 2^-8."""
import pytest
import torch

import ops_reference as ref
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
@pytest.mark.parametrize("cols", [(1 << 21) - 3, (1 << 21) + 77, 3 * (1 << 21) + 5])
def test_wide_rows(rt, dtype, cols):
    t = DTYPES[dtype]
    gen = torch.Generator(device="cuda").manual_seed(cols)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(t)  # noqa: E731
    x, dy, g = rnd(2, cols), rnd(2, cols), rnd(cols)
    _, mean, rstd = rt.layer_norm(x, g, g)
    dx, dg, db = rt.layer_norm_backward(dy, x, g, mean, rstd)
    half = E16 if t == torch.bfloat16 else 0.0
    edx, edg, edb = ref.norm_backward(dy.double(), x.double(), g.double(), mean.double(), rstd.double())
    xh = (x.double() - mean.double()[:, None]) * rstd.double()[:, None]
    a = (dy.double() * g.double()).abs()
    sums = (cols / 256 + 16) * E32
    tol = rstd.double()[:, None] * ((a + a.mean(1, keepdim=True) + xh.abs() * (a * xh.abs()).mean(1, keepdim=True)) * 8 * E32
                                    + sums * (a.mean(1, keepdim=True) + xh.abs() * (a * xh.abs()).mean(1, keepdim=True)))
    within(dx.double() - edx, tol + half * edx.abs(), "dx")
    # (xh itself: a difference, a product; x - mean may cancel)
    slack = (dy.double().abs() * (xh.abs() + (x.double().abs() + mean.double().abs()[:, None]) * rstd.double()[:, None])).sum(0)
    within(dg.double() - edg, 4 * E32 * slack + half * edg.abs(), "dg")
    within(db.double() - edb, 2 * E32 * dy.double().abs().sum(0) + half * edb.abs(), "db")


def test_refused(rt):
    from paper_2604_15380_amd import binding as B
    a = torch.zeros(8, device="cuda").data_ptr()
    for cols in ((1 << 30) + 1, (1 << 31) - 1):
        with pytest.raises(B.PainnError) as e:
            B.painn_layer_norm(rt.ctx, 1, 1, cols, a, cols, a, a, 1e-5, a, cols, None, None)
        assert e.value.status == -8
        with pytest.raises(B.PainnError) as e:
            B.painn_layer_norm_backward(rt.ctx, 1, 1, cols, a, cols, a, cols, a, a, a, None, 0, a, a)
        assert e.value.status == -8
