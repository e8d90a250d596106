"""AdamW with 8-bit states beside 32-bit ones over many steps.

Codes are rounded to nearest at every step, so most second moments move only
with their block's scale.  The bounds are those that painn.h states, from CPU
runs of its formula with other seeds (sqrt(v) within 0.54 to 1.95 of 32 bits
after 1,000 to 4,000 steps; the parameters' way 0.25 of itself apart at most),
widened by a third."""
import pytest
import torch

pytestmark = pytest.mark.gpu

N = 256 * 16


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


@pytest.mark.parametrize("spread", [0.0, 0.7])
def test_beside_32_bits(rt, spread):
    gen = torch.Generator(device="cuda").manual_seed(77)
    size = torch.exp(spread * torch.randn(N, generator=gen, device="cuda"))
    g = torch.zeros(N, device="cuda")
    p, q = torch.zeros(N, device="cuda"), torch.zeros(N, device="cuda")
    how = dict(lr=1e-3, weight_decay=0.0)
    a, b = rt.adamw([p], [g], state_bits=8, **how), rt.adamw([q], [g], **how)

    def steps(n, scale):
        for _ in range(n):
            g.copy_(torch.randn(N, generator=gen, device="cuda") * size * scale)
            a.step()
            b.step()

    def held():
        r = a.v[0].float().view(-1, 256) * a.v_scale[0][:, None]
        return (r.view(-1) / b.v[0].sqrt()).double()

    steps(1200, 1.0)
    ratio = held()
    assert 0.54 / 1.33 < float(ratio.min()) and float(ratio.max()) < 1.95 * 1.33
    assert 0.67 / 1.33 < float(ratio.quantile(0.05)) and float(ratio.quantile(0.95)) < 1.5 * 1.33
    assert float((p - q).norm()) < 0.25 * 1.33 * float(q.norm())
    # gradients that become small in a whole block take its scale along
    steps(1200, 0.01)
    later = held()
    assert 0.54 / 1.33 < float(later.min()) and float(later.max()) < 1.95 * 1.33
    assert bool(p.isfinite().all())
    a.free()
    b.free()
