"""The gate where many heads meet many rows: several blocks of long rows, with
the largest heads found one by one or by counting."""
import pytest
import torch

import gate_norm_reference as R
import test_gpu_gate as G

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


@pytest.mark.parametrize("dtype", list(G.DTYPES))
@pytest.mark.parametrize("rows,heads,k", [(4200, 1000, 5), (4100, 1024, 12), (66000, 16, 9), (140001, 7, 3)])
def test_both_passes(rt, dtype, rows, heads, k):
    t = G.DTYPES[dtype]
    x, _, gen = G.inputs(rows, heads, t, 77, True)
    dw = torch.randn(rows, k, generator=gen)
    got = rt.gate(x.cuda(), k)
    idx, counts, some = G.check_forward(x, k, False, got)
    d = rt.gate_backward(dw.cuda(), x.cuda(), got, balance=0.3)
    G.check_backward(x, dw, idx, counts, some, False, 0.3, d, t)
