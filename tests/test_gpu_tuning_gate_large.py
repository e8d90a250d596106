"""GateTuner where total energies are large beside what the heads differ by: its
loss and its gradients against 64 bits."""
import pytest
import torch

import gate_norm_reference as R
import ops_reference as ref
from test_gpu_tuning_gate import done, gate_setup

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


def exact(tuner, b, target):
    """Loss, and by name the gradients and the sums of their terms' magnitudes,
    in 64 bits.  A slope of SiLU is 1.1 at most."""
    w = {k: v.double().cpu() for k, v in tuner.master.items()}
    x, e, t = b["x"].double().cpu(), b["heads"].cpu(), target.cpu()
    inputs, zs = [], []
    for m in range(3):
        inputs.append(x)
        zs.append(x @ w[f"blend{m}.w"].t() + w[f"blend{m}.b"])
        x = ref.act(zs[-1], "silu") if m < 2 else zs[-1]
    weights, idx, counts, share, balance, rows, p = R.gate(x, tuner.k, tuner.normalize)
    own = e.gather(1, idx.long())
    blended = (weights * own).sum(1)
    diff = blended - t
    d = 2 / len(x) * diff[:, None] * own
    dx, _ = R.gate_backward(x, d, idx, counts, rows, tuner.normalize, tuner.balance)
    # what the terms cannot do without: the heads' distance from the blend where weights add up to 1
    if tuner.normalize or tuner.k == tuner.n_heads:
        d = 2 / len(x) * diff[:, None] * (own - blended[:, None])
    _, mag = R.gate_backward(x, d, idx, counts, rows, tuner.normalize, tuner.balance)
    out = {}
    for m in (2, 1, 0):
        out[f"blend{m}.w"] = dx.t() @ inputs[m], mag.t() @ inputs[m].abs()
        out[f"blend{m}.b"] = dx.sum(0), mag.sum(0)
        if m:
            dx = (dx @ w[f"blend{m}.w"]) * ref.slope(zs[m - 1], "silu")
            mag = 1.1 * (mag @ w[f"blend{m}.w"].abs())
    return (diff ** 2).mean() + tuner.balance * balance, idx, out


@pytest.mark.parametrize("k,normalize,level", [(None, False, 0.0), (2, False, 0.0), (None, False, 1e3), (None, False, 1e5),
                                               (2, True, 1e5), (5, True, 1e4), (None, True, 1e5)])
def test_large_energies(rt, k, normalize, level):
    """Heads 0.1 apart at energies of `level`.  A few hundred rounded terms leave
    2e-5 of the terms' magnitudes, which do not have the level in them (FP64
    leaves 2^-53 of 1e5 there, 1e-10 of 0.1)."""
    hp, W, batch, model, graph, heads, tuner, _ = gate_setup(rt, k=k, normalize=normalize)
    gen = torch.Generator(device="cuda").manual_seed(16)
    n = batch.n_struct
    normal = lambda *s: torch.randn(*s, generator=gen, device="cuda", dtype=torch.float64)  # noqa: E731
    heads = level * (1 + 0.2 * normal(n, 1)) + 0.1 * normal(n, hp.n_heads)
    b = tuner.batch(batch.species, batch.struct_ptr, heads)
    target = heads.mean(1) + 0.2 * normal(n)
    loss = tuner.gradients(b, target)
    want, idx, grads = exact(tuner, b, target)
    assert torch.equal(idx, tuner.gate.indices.cpu())
    assert abs(float(loss) / float(want) - 1) < 2e-5
    for name, (g, mag) in grads.items():
        off = (tuner.grad[name].double().cpu() - g).abs()
        assert bool((off <= 2e-5 * mag).all()), (name, float((off / mag).max()))
    done(tuner, graph, model)


def test_one_head_has_no_gradient(rt):
    """The weight of a single normalised head is 1 whatever the logits."""
    hp, W, batch, model, graph, heads, tuner, _ = gate_setup(rt, k=1, normalize=True)
    b = tuner.batch(batch.species, batch.struct_ptr, heads + 1e5)
    tuner.gradients(b, heads[:, 0] + 1e5 - 3.0)
    assert not any(bool(g.any()) for g in tuner.grad.values())
    done(tuner, graph, model)
