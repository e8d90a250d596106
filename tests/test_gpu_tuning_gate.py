"""The tuners with the gate, group norm and clipping put together: GateTuner
starts as the library's own blend, HeadTuner with a group-norm adapter as the
model it is given; their FP32 gradients are checked against directional
differences of 64-bit copies, and a clipped step's against AdamW on the
clipped gradients."""
import numpy as np
import pytest
import torch

import gate_norm_reference as R
import ops_reference as ref
import synth
from test_gpu_tuning import setup as head_setup

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


def gate_setup(rt, **how):
    from paper_2604_15380_amd.tuning import GateTuner, head_energies
    hp = synth.HyperParams(F=64, K=20, L=2, n_species=85, n_heads=6, cutoff=5.0, shared_dims=[50],
                           branch_dims=[40, 1], blend_dims=[24, 16])
    W = synth.make_weights(hp, 33)
    batch = synth.make_batch("screening", 0, 60)
    model = rt.load_model(synth.weight_file_bytes(hp, W))
    graph = rt.build_graph(rt.upload_batch(batch), hp.cutoff)
    heads = head_energies(rt, model, graph, "fp64")
    tuner = GateTuner(rt, W, 3, **how)
    return hp, W, batch, model, graph, heads, tuner, tuner.batch(batch.species, batch.struct_ptr, heads)


def done(*objects):
    for o in objects:
        o.free()


@pytest.mark.parametrize("dtype,tol", [("fp32", 1e-5), ("bf16", 2e-2)])
def test_starts_as_the_blend(rt, dtype, tol):
    """Bound: the library's energy tolerance of the precision, twice, of the sum
    of the heads' |E| (in BF16 the softmax's too, whose logits are rounded)."""
    hp, W, batch, model, graph, heads, tuner, b = gate_setup(rt, dtype=dtype)
    weights = torch.empty(batch.n_struct, hp.n_heads, dtype=torch.float64, device="cuda")
    want = rt.forward_blend(model, graph, dtype, weights=weights)
    got = tuner.energies(b)
    size = heads.abs().sum(1)
    assert bool(((got - want).abs() <= 2 * tol * size).all())
    done(tuner, graph, model)


def loss64(tuner, b, weights, target):
    """The loss in 64 bits from the masters; the choices and counts come with it."""
    x = b["x"].double().cpu()
    for m in range(3):
        x = x @ weights[f"blend{m}.w"].double().cpu().t() + weights[f"blend{m}.b"].double().cpu()
        if m < 2:
            x = ref.act(x, "silu")
    w, idx, counts, share, loss, rows, p = R.gate(x, tuner.k, tuner.normalize)
    e = b["heads"].cpu().gather(1, idx.long().clamp_min(0)) * (idx >= 0)
    return float((((w * e).sum(1) - target.cpu()) ** 2).mean() + tuner.balance * loss), idx


@pytest.mark.parametrize("k,normalize", [(None, False), (2, True)])
def test_gate_gradient_against_differences(rt, k, normalize):
    """A few hundred rounded terms per value leave 2e-5 of the terms' magnitudes,
    as in the heads' own test."""
    hp, W, batch, model, graph, heads, tuner, b = gate_setup(rt, k=k, normalize=normalize, balance=0.5)
    gen = torch.Generator(device="cuda").manual_seed(6)
    target = heads.mean(1) + torch.randn(batch.n_struct, generator=gen, device="cuda", dtype=torch.float64)
    loss = tuner.gradients(b, target)
    base, idx = loss64(tuner, b, tuner.master, target)
    assert torch.equal(idx, tuner.gate.indices.cpu())
    assert abs(float(loss) / base - 1) < 1e-5
    h = 1e-6
    for name, w in tuner.master.items():
        u = torch.randn(w.shape, generator=gen, device="cuda", dtype=torch.float64)
        ends = []
        for sgn in (1, -1):
            moved = {n: (v.double() + sgn * h * u if n == name else v) for n, v in tuner.master.items()}
            value, other = loss64(tuner, b, moved, target)
            assert torch.equal(other, idx)
            ends.append(value)
        num = (ends[0] - ends[1]) / (2 * h)
        g = tuner.grad[name].double()
        assert abs(num - float((g * u).sum())) <= 2e-5 * float((g * u).abs().sum()) + 1e-7 * base, name
    done(tuner, graph, model)


@pytest.mark.parametrize("dtype,bits,k", [("fp32", 32, None), ("bf16", 8, 2)])
def test_gate_steps(rt, dtype, bits, k):
    """Steps run, change every array, clip, and give weights for the model's file."""
    hp, W, batch, model, graph, heads, tuner, b = gate_setup(rt, dtype=dtype, state_bits=bits, k=k, balance=0.1,
                                                             max_norm=0.5, lr=1e-2)
    before = {n: v.clone() for n, v in tuner.master.items()}
    target = heads[:, 3].clone()
    losses = [float(tuner.step(b, target)) for _ in range(10)]
    assert all(np.isfinite(losses)) and float(tuner.norm) > 0
    assert all(not torch.equal(before[n], v) for n, v in tuner.master.items())
    out = tuner.weights()
    assert set(out) == {n for n, _ in synth.weight_layout(hp) if n.startswith("blend")}
    again = rt.load_model(synth.weight_file_bytes(hp, {**W, **out}))
    if dtype == "fp32":
        want = rt.forward_blend(again, graph, "fp32")
        assert bool(((tuner.energies(b) - want).abs() <= 2e-5 * heads.abs().sum(1)).all())
    done(tuner, again, graph, model)


def test_a_clipped_step(rt):
    """One step with max_norm is a step of AdamW on the gradients times the
    factor; a large max_norm changes nothing."""
    made = []
    for max_norm in (None, 0.25, 1e30):
        *rest, s, tuner = head_setup(rt, "fp32", 0, max_norm=max_norm)
        hp, W, batch, model, graph, inp = rest
        b = tuner.batch(s, batch.struct_ptr, batch.dataset_id)
        tuner.step(b, 0.0)
        made.append((tuner, model, graph))
    plain, clipped, loose = (m[0] for m in made)
    assert all(torch.equal(plain.master[k], loose.master[k]) for k in plain.master)
    norm = torch.sqrt(sum((g.double() ** 2).sum() for g in clipped.grad.values()))
    assert float(clipped.norm) == pytest.approx(float(norm), rel=1e-6) and float(norm) > 0.25
    # m after one step is 0.1 of the gradient
    for m, (name, g) in zip(clipped.optimizer.m, clipped.grad.items()):
        want = g.double().view(-1) * (0.25 / float(norm)) * 0.1
        assert bool(((m.double().view(-1) - want).abs() <= 4e-7 * want.abs() + 1e-30).all()), name
    for tuner, model, graph in made:
        done(tuner, model, graph)


@pytest.mark.parametrize("dtype,tol", [("fp32", 1e-5), ("bf16", 2e-2)])
def test_group_norm_adapter_starts_as_the_model(rt, dtype, tol):
    hp, W, batch, model, graph, inp, s, tuner = head_setup(rt, dtype, 96, adapter_norm="group", adapter_groups=12)
    s, _ = rt.features(model, graph, hp.L - 1, dtype)
    b = tuner.batch(s, batch.struct_ptr, batch.dataset_id)
    mine = tuner.energies(b)
    own = rt.forward(model, graph, dtype, inp["dataset_id"])
    size = rt.forward(model, graph, "fp64", inp["dataset_id"]).abs() + torch.as_tensor(np.diff(batch.struct_ptr)).cuda()
    assert bool(((mine - own).abs() <= 4 * tol * size).all())
    done(tuner, graph, model)


def test_group_norm_adapter_gradient(rt):
    hp, W, batch, model, graph, inp, s, tuner = head_setup(rt, "fp32", 96, adapter_norm="group", adapter_groups=12)
    gen = torch.Generator(device="cuda").manual_seed(7)
    tuner.master["adapter1.w"].normal_(0, 0.05, generator=gen)
    b = tuner.batch(s, batch.struct_ptr, batch.dataset_id)
    target = torch.randn(batch.n_struct, generator=gen, device="cuda", dtype=torch.float64) * 3
    ptr, cuts = b["ptr"].tolist(), b["offsets"].tolist()

    def loss64(weights):
        w = {k: v.cpu().double() for k, v in weights.items()}
        x = b["s"].cpu().double()
        t = x @ w["adapter0.w"].t() + w["adapter0.b"]
        h = R.group_norm(t, w["norm.w"], w["norm.b"], 12, list(zip(ptr[:-1], ptr[1:])), 1e-5, "silu")[0]
        x = x + h @ w["adapter1.w"].t() + w["adapter1.b"]
        for m in range(2):
            x = ref.act(x @ w[f"shared{m}.w"].t() + w[f"shared{m}.b"], "silu")
        e = torch.zeros(len(x), dtype=torch.float64)
        for k in range(tuner.n_heads):
            y = x[cuts[k]:cuts[k + 1]]
            for m in range(3):
                y = y @ w[f"branch{m}.w"][k].t() + w[f"branch{m}.b"][k]
                y = ref.act(y, "silu") if m < 2 else y
            e[cuts[k]:cuts[k + 1]] = y[:, 0]
        E = torch.stack([e[a:c].sum() for a, c in zip(ptr[:-1], ptr[1:])])
        return float((E - target.cpu()).abs().mean())

    loss = tuner.gradients(b, target)
    assert abs(float(loss) / loss64(tuner.master) - 1) < 1e-5
    h = 1e-5
    for name in ("adapter0.w", "adapter0.b", "norm.w", "norm.b", "adapter1.w", "adapter1.b", "shared0.w"):
        w = tuner.master[name]
        u = torch.randn(w.shape, generator=gen, device="cuda", dtype=torch.float64)
        ends = [loss64({n: (v.double() + sgn * h * u if n == name else v) for n, v in tuner.master.items()})
                for sgn in (1, -1)]
        num = (ends[0] - ends[1]) / (2 * h)
        g = tuner.grad[name].double()
        assert abs(num - float((g * u).sum())) <= 2e-5 * float((g * u).abs().sum()) + 1e-8, name
    for _ in range(3):
        assert np.isfinite(float(tuner.step(b, target)))
    done(tuner, graph, model)


def test_refusals(rt):
    from paper_2604_15380_amd.tuning import GateTuner
    with pytest.raises(ValueError):
        head_setup(rt, "fp32", 96, adapter_norm="batch")
    with pytest.raises(ValueError):
        head_setup(rt, "fp32", 96, adapter_norm="group", adapter_groups=7)
    hp, W, batch, model, graph, heads, tuner, b = gate_setup(rt)
    for k in (0, 7):
        with pytest.raises(ValueError):
            GateTuner(rt, W, 3, k=k)
    with pytest.raises(ValueError):
        GateTuner(rt, W, 3, dtype="fp64")
    with pytest.raises(ValueError):
        tuner.batch(batch.species, batch.struct_ptr, heads[:, :5])
    with pytest.raises(ValueError):
        tuner.batch(batch.species + 85, batch.struct_ptr, heads)
    with pytest.raises(ValueError):
        tuner.gradients(b, torch.zeros(3, device="cuda"))
    done(tuner, graph, model)
