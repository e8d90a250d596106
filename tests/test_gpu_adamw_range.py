"""AdamW's hyperparameters at the ends of FP32, in which the step is computed:
what it cannot hold is refused, what it can moves no value without gradient to
NaN."""
import pytest
import torch

pytestmark = pytest.mark.gpu

FLT_MAX = float(torch.finfo(torch.float32).max)


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_refused(rt, bits):
    from paper_2604_15380_amd import PainnError
    p, g = torch.ones(300, device="cuda"), torch.zeros(300, device="cuda")
    for kw in (dict(eps=1e-50), dict(eps=1e39), dict(weight_decay=1e39), dict(steps=(1 << 62) + 1)):
        with pytest.raises(PainnError) as e:
            rt.adamw([p], [g], state_bits=bits, **kw)
        assert e.value.status == -1, kw
    opt = rt.adamw([p], [g], state_bits=bits, weight_decay=1e30)
    for lr in (1e39, 1e38, 1e10):       # lr itself; lr / (1 - 0.9); lr times 1e30
        with pytest.raises(PainnError) as e:
            opt.step(lr)
        assert e.value.status == -1, lr
    assert opt.steps == 0
    torch.cuda.synchronize()
    assert bool((p == 1).all())
    opt.free()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("eps", [1e-44, 1e-30, 1e38])
def test_no_gradient_no_movement(rt, bits, eps):
    p, g = torch.ones(300, device="cuda"), torch.zeros(300, device="cuda")
    opt = rt.adamw([p], [g], state_bits=bits, eps=eps, weight_decay=0.0, steps=1 << 62)
    for lr in (1e-3, FLT_MAX, 0.0):
        opt.step(lr)
    torch.cuda.synchronize()
    assert bool((p == 1).all()) and opt.steps == (1 << 62) + 3
    opt.free()
