"""Sizes beyond one launch (2^32 threads along its axis) are refused before
anything is launched or allocated; no array of such a size is needed."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("sizes", [[1 << 34], [1 << 33, (1 << 33) - 1023], [1 << 62]])
def test_adamw(rt, bits, sizes):
    """2^24 - 1 blocks of 1,024 values: 2^34 - 1,024 of one tensor."""
    from paper_2604_15380_amd import binding as B
    a = torch.zeros(8, device="cuda").data_ptr()
    cfg = dict(beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, state_bits=bits, grad_precision=1, steps=0)
    tensors = [dict(n=n, param=a, grad=a, m=a, v=a, m_scale=a, v_scale=a) for n in sizes]
    with pytest.raises(B.PainnError) as e:
        B.painn_adamw_create(rt.ctx, tensors, cfg)
    assert e.value.status == -8


@pytest.mark.parametrize("precision", [1, 2])
@pytest.mark.parametrize("rows,width", [(1 << 33, 1), (1 << 31, 256), (1 << 40, 1 << 20)])
def test_dense(rt, precision, rows, width):
    """Tiles of at most 256 rows and columns, 256 threads each at least."""
    from paper_2604_15380_amd import binding as B
    a = torch.zeros(8, device="cuda").data_ptr()
    fwd = dict(precision=precision, activation=1, rows=rows, d_in=1, d_out=width, x=a, ldx=1, w=a, y=a, ldy=width)
    back = dict(precision=precision, activation=0, rows=rows, d_in=width, d_out=1, dy=a, lddy=1, w=a, dx=a, lddx=width)
    with pytest.raises(B.PainnError) as e:
        B.painn_linear(rt.ctx, B.painn_linear_args(**fwd))
    assert e.value.status == -8
    with pytest.raises(B.PainnError) as e:
        B.painn_linear_backward(rt.ctx, B.painn_linear_backward_args(**back))
    assert e.value.status == -8
