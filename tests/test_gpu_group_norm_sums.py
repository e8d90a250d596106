"""dgamma and dbeta of group norm in FP32: sums of terms of one sign.

x and dy have 8 digits, the mean is 0 and rstd 1, so that every term is exact, and
all are positive: a sum that is formed in FP64 but for one rounding per block and
the result's is off by 2 E32 of itself, however many rows there are."""
import pytest
import torch

from ops_reference import E32, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


# few long samples, samples of a block of 512 and 256, of a wave, and single ones
@pytest.mark.parametrize("rows,cols,groups,samples", [(120000, 192, 8, 5), (147456, 256, 32, 144), (65536, 64, 4, 512),
                                                      (65520, 250, 10, 1820), (100000, 40, 5, 100000), (400, 2048, 1, 1)])
def test_terms_of_one_sign(rt, rows, cols, groups, samples):
    gen = torch.Generator(device="cuda").manual_seed(rows)
    x, dy = ((0.5 + torch.rand(rows, cols, generator=gen, device="cuda")).bfloat16().float() for _ in range(2))
    mean, rstd = torch.zeros(samples, groups, device="cuda"), torch.ones(samples, groups, device="cuda")
    one = torch.ones(cols, device="cuda")
    _, dg, db = rt.group_norm_backward(dy, x, one, one, mean, rstd, groups, sample_rows=rows // samples)
    for got, terms, name in ((dg, dy.double() * x.double(), "dgamma"), (db, dy.double(), "dbeta")):
        want = terms.sum(0)
        within(got.double() - want, 2.01 * E32 * want, name)
