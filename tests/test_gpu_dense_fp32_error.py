"""FP32 products over BF16 planes are at least as near to 64 bits as a plain
FP32 product of the same operands (torch's on the same GPU), in the 2-norm, for
values of either sign and for positive ones, whose sums grow with every term."""
import pytest
import torch

pytestmark = pytest.mark.gpu

SHAPES = [(1, 776, 776), (16, 776, 776), (64, 776, 64), (40, 300, 1024), (200, 50, 776), (4096, 337, 776),
          (4096, 64, 256), (9000, 776, 128)]


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


def off(a, exact):
    return float((a.double() - exact).norm() / exact.norm())


@pytest.mark.parametrize("positive", [False, True])
@pytest.mark.parametrize("n,i,o", SHAPES)
def test_no_further_than_fp32(rt, n, i, o, positive):
    gen = torch.Generator(device="cuda").manual_seed(i + positive)
    draw = torch.rand if positive else torch.randn
    x, w, dy = (draw(*s, generator=gen, device="cuda") for s in ((n, i), (o, i), (n, o)))
    dx, dw, _ = rt.linear_backward(dy, x, w)
    for what, mine, plain, exact in (
            ("y", rt.linear(x, w), x @ w.t(), x.double() @ w.double().t()),
            ("dx", dx, dy @ w, dy.double() @ w.double())):
        assert off(mine, exact) <= off(plain, exact), (what, off(mine, exact), off(plain, exact))
