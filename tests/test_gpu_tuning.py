"""HeadTuner: the head-tuning operators put together.

The tuner starts as the model it is given, so its energies are the library's
own of the same precision (bounds: the library's energy tolerances, FP32 1e-5
and BF16 2e-2 of the sum of |e_i|, twice, for two computations).  Its gradient
in FP32 is checked against directional differences of a 64-bit copy of the
heads, and steps lower the loss."""
import numpy as np
import pytest
import torch

import ops_reference as ref
import synth

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


def setup(rt, dtype, adapter, **how):
    from paper_2604_15380_amd.tuning import HeadTuner, dataset_order
    hp = synth.HyperParams(F=64, K=20, L=2, n_species=85, n_heads=5, cutoff=5.0, shared_dims=[50, 50],
                           branch_dims=[72, 40, 1])
    W = synth.make_weights(hp, 31)
    b = synth.make_batch("screening", 0, 60)
    b.dataset_id[:] = b.dataset_id % 4          # one head without rows
    b = b.subset(dataset_order(b.dataset_id))
    model = rt.load_model(synth.weight_file_bytes(hp, W))
    inp = rt.upload_batch(b)
    graph = rt.build_graph(inp, hp.cutoff)
    s, _ = rt.features(model, graph, hp.L - 1, "fp64")
    tuner = HeadTuner(rt, W, hp.F, hp.n_heads, 2, 3, dtype=dtype, adapter=adapter, **how)
    return hp, W, b, model, graph, inp, s, tuner


def atom_energies(tuner, s, b, weights):
    """Atom energies of the tuner's network in 64 bits."""
    w = {k: v.cpu().double() for k, v in weights.items()}
    x = s.cpu().double()
    if tuner.adapter:
        h, _, _ = ref.norm(x, w["norm.w"], w["norm.b"], 1e-5)
        t = ref.act(h @ w["adapter0.w"].t() + w["adapter0.b"], "silu")
        x = x + t @ w["adapter1.w"].t() + w["adapter1.b"]
    for m in range(2):
        x = ref.act(x @ w[f"shared{m}.w"].t() + w[f"shared{m}.b"], "silu")
    out = torch.zeros(len(x), dtype=torch.float64)
    cuts = b["offsets"].tolist()
    for h in range(tuner.n_heads):
        y = x[cuts[h]:cuts[h + 1]]
        for m in range(3):
            y = y @ w[f"branch{m}.w"][h].t() + w[f"branch{m}.b"][h]
            if m < 2:
                y = ref.act(y, "silu")
        out[cuts[h]:cuts[h + 1]] = y[:, 0]
    return out


def loss64(tuner, s, b, weights, target):
    e = atom_energies(tuner, s, b, weights)
    ptr = b["ptr"].tolist()
    E = torch.stack([e[a:c].sum() for a, c in zip(ptr[:-1], ptr[1:])])
    return float((E - target.cpu()).abs().mean())


@pytest.mark.parametrize("dtype,tol", [("fp32", 1e-5), ("bf16", 2e-2)])
@pytest.mark.parametrize("adapter", [0, 96])
def test_starts_as_the_model(rt, dtype, tol, adapter):
    hp, W, batch, model, graph, inp, s, tuner = setup(rt, dtype, adapter)
    prec = dtype
    s, _ = rt.features(model, graph, hp.L - 1, prec)
    b = tuner.batch(s, batch.struct_ptr, batch.dataset_id)
    mine = tuner.energies(b).cpu()
    own = rt.forward(model, graph, prec, inp["dataset_id"]).cpu()
    e = atom_energies(tuner, s, b, tuner.master).abs()
    ptr = batch.struct_ptr
    size = torch.stack([e[a:c].sum() for a, c in zip(ptr[:-1], ptr[1:])])
    assert bool(((mine - own).abs() <= 2 * tol * size).all())
    tuner.free()
    graph.free()
    model.free()


def test_gradient_against_differences(rt):
    """The FP32 gradient of every array along a random direction against a
    central difference of the 64-bit loss: a few hundred rounded terms per
    value leave 1e-5 of the terms' magnitudes, the difference 1e-8."""
    hp, W, batch, model, graph, inp, s, tuner = setup(rt, "fp32", 96)
    gen = torch.Generator(device="cuda").manual_seed(5)
    tuner.master["adapter1.w"].normal_(0, 0.05, generator=gen)      # (an adapter that does something)
    b = tuner.batch(s, batch.struct_ptr, batch.dataset_id)
    target = torch.randn(batch.n_struct, generator=gen, device="cuda", dtype=torch.float64) * 3
    loss = tuner.gradients(b, target)
    s32 = b["s"]
    assert abs(float(loss) / loss64(tuner, s32, b, tuner.master, target) - 1) < 1e-5
    h = 1e-5
    for k, w in tuner.master.items():
        u = torch.randn(w.shape, generator=gen, device="cuda", dtype=torch.float64)
        ends = []
        for sgn in (1, -1):
            moved = {n: (v.double() + sgn * h * u if n == k else v) for n, v in tuner.master.items()}
            ends.append(loss64(tuner, s32, b, moved, target))
        num = (ends[0] - ends[1]) / (2 * h)
        g = tuner.grad[k].double()
        assert abs(num - float((g * u).sum())) <= 2e-5 * float((g * u).abs().sum()) + 1e-9, k
    assert not bool(tuner.grad["branch0.w"][4].any())            # the head without rows
    tuner.free()
    graph.free()
    model.free()


@pytest.mark.parametrize("dtype,bits", [("fp32", 32), ("bf16", 32), ("bf16", 8)])
def test_steps_lower_the_loss(rt, dtype, bits):
    """Targets are another head set's energies plus an offset per dataset;
    thirty steps take the loss below a half of the first."""
    hp, W, batch, model, graph, inp, s, tuner = setup(rt, dtype, 96, lr=3e-3, state_bits=bits)
    b = tuner.batch(s, batch.struct_ptr, batch.dataset_id)
    shift = torch.tensor(np.array([3.0, -2.0, 5.0, 1.0, 0.0])[batch.dataset_id], device="cuda")
    atoms = (b["ptr"][1:] - b["ptr"][:-1]).double()
    target = tuner.energies(b) + 0.05 * shift * atoms
    losses = [float(tuner.step(b, target)) for _ in range(30)]
    assert all(np.isfinite(losses)) and losses[-1] < 0.5 * losses[0], losses
    out = tuner.weights()
    assert set(out) == {n for n, _ in synth.weight_layout(hp) if n.startswith(("shared", "head"))}
    assert all(out[n].shape == W[n].shape for n in out)
    tuner.free()
    graph.free()
    model.free()


def test_refusals(rt):
    hp, W, batch, model, graph, inp, s, tuner = setup(rt, "fp32", 0)
    with pytest.raises(ValueError):
        tuner.batch(s[:-1], batch.struct_ptr, batch.dataset_id)
    with pytest.raises(ValueError):
        tuner.batch(s, batch.struct_ptr, batch.dataset_id[::-1].copy())
    with pytest.raises(ValueError):
        tuner.batch(s, batch.struct_ptr, batch.dataset_id + 3)
    from paper_2604_15380_amd.tuning import HeadTuner
    with pytest.raises(ValueError):
        HeadTuner(rt, W, hp.F, hp.n_heads, 2, 3, dtype="fp64")
    tuner.free()
    graph.free()
    model.free()
