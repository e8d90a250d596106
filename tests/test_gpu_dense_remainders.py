"""The reverse pass of BF16 layers whose dz keeps its remainders by request, at
sizes where it is rounded otherwise: the bounds of
test_few_values_of_dz_are_not_rounded."""
import pytest
import torch

import ops_reference as ref
from ops_reference import E16, E32, sum_bound, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


def ragged(n, groups):
    cuts = [0] + [int(n * ((k + 1) / groups) ** 2.5) for k in range(groups)]
    cuts[3] = cuts[4]
    cuts[-1] = n
    return cuts


@pytest.mark.parametrize("n,i,o,groups", [(8193, 40, 1, 0), (300, 130, 200, 0), (129, 72, 64, 0), (20000, 776, 776, 16),
                                          (20000, 337, 50, 5), (65502, 256, 264, 0)])
@pytest.mark.parametrize("x_act", ["none", "silu"])
def test_kept(rt, n, i, o, groups, x_act):
    gen = torch.Generator(device="cuda").manual_seed(n + i)
    mk = lambda *s, scale=1.0: (torch.randn(*s, generator=gen, device="cuda") * scale).bfloat16()  # noqa: E731
    G = groups or 1
    cuts = ragged(n, groups) if groups else [0, n]
    dy, z, x, xz, w = mk(n, o), mk(n, o, scale=2.0), mk(n, i), mk(n, i, scale=2.0), mk(G, o, i, scale=o ** -0.5)
    ranges = ref.spans(cuts, n)
    r = ref.linear_backward(dy.double(), z.double(), "silu", x.double(), w.double(), xz.double(), x_act, ranges)
    how = dict(activation="silu", preact=z, x_activation=x_act, x_preact=xz if x_act != "none" else None)
    if groups:
        off = torch.tensor(cuts, dtype=torch.int32, device="cuda")
        run = lambda **k: rt.grouped_linear_backward(dy, x, w, off, **how, **k)  # noqa: E731
    else:
        run = lambda **k: rt.linear_backward(dy, x, w[0], **how, **k)  # noqa: E731
    got, rounded = run(dz_remainders=True), run()
    rows = max(b - a for a, b in ranges)
    for name, mine, other, k in zip(("dx", "dw"), got, rounded, (o, rows)):
        mine, other = (a.double().reshape(r[name].shape) for a in (mine, other))
        tol = (sum_bound(2 * k) + E16 * E16) * r["m" + name] + 16 * E32 * r["e" + name] + E16 * r[name].abs()
        within(mine - r[name], tol, name)
        # nearer than with one rounding of dz, whose error adds to the result's
        err = lambda a: float((a - r[name]).norm())  # noqa: E731
        assert err(mine) < 0.9 * err(other), (name, err(mine), err(other))
    assert torch.equal(got[2], rounded[2])          # dbias has never been rounded
    again = run(dz_remainders=True)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_no_activation_and_fp32_have_none(rt):
    x, dy, w = (torch.randn(*s, device="cuda") for s in ((500, 40), (500, 72), (72, 40)))
    for t in (torch.float32, torch.bfloat16):
        a, b, c = x.to(t), dy.to(t), w.to(t)
        assert all(torch.equal(p, q) for p, q in zip(rt.linear_backward(b, a, c), rt.linear_backward(b, a, c, dz_remainders=True)))
    got = rt.linear_backward(dy, x, w, activation="silu", preact=dy, dz_remainders=True)
    assert all(torch.equal(p, q) for p, q in zip(got, rt.linear_backward(dy, x, w, activation="silu", preact=dy)))


def test_refusal(rt):
    from paper_2604_15380_amd import PainnError
    x, dy, w = (torch.zeros(*s, device="cuda") for s in ((5, 4), (5, 7), (7, 4)))
    for bad in (2, -1):
        with pytest.raises(PainnError) as e:
            rt.linear_backward(dy, x, w, dz_remainders=bad)
        assert e.value.status == -1
