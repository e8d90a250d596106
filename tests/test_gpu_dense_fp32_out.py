"""FP32 results of BF16 dense layers (a readout's energies) against the 64-bit
form: the bounds of test_gpu_dense.py without the rounding of the result; and
HeadTuner's atom energies, which take them.

The readout's sum bound at 72 terms is 42 2^-24 of the magnitudes, a hundredth
of what a BF16 result's rounding may leave."""
import pytest
import torch

import ops_reference as ref
from ops_reference import E16, E32, sum_bound, within
from test_gpu_tuning import rt, setup  # noqa: F401

pytestmark = pytest.mark.gpu


def maker(seed):
    g = torch.Generator().manual_seed(seed)
    return lambda *s, scale=1.0: (torch.randn(*s, generator=g) * scale).bfloat16()


@pytest.mark.parametrize("n,i,o,offsets", [(1, 776, 1, None), (30, 776, 1, None), (300, 64, 1, None),
                                           (300, 57, 3, [0, 7, 7, 150, 290]), (40, 264, 8, [0, 1, 1, 40]),
                                           (5000, 776, 1, [0, 2000, 2000, 4999, 5000]), (20000, 50, 1, None),
                                           (2000, 128, 200, None), (129, 45, 37, None)])
@pytest.mark.parametrize("kind,residual", [("none", False), ("gelu", True)])
def test_forward(rt, n, i, o, offsets, kind, residual):  # noqa: F811
    mk = maker(n + i)
    G = len(offsets) - 1 if offsets else 1
    x, w, b, r = mk(n, i), mk(G, o, i, scale=i ** -0.5), mk(G, o), mk(n, o)
    ranges = ref.spans(offsets, n) if offsets else [(0, n)]
    yr, zr, mag = ref.linear(x.double(), w.double(), b.double(), kind, r.double() if residual else None, ranges)
    base = torch.full((n, o + 3), 7.0, device="cuda")
    how = dict(activation=kind, residual=r.cuda() if residual else None, keep_preact=True, out=base[:, :o])
    if offsets:
        off = torch.tensor(offsets, dtype=torch.int32).cuda()
        y, z = rt.grouped_linear(x.cuda(), w.cuda(), off, b.cuda(), **how)
    else:
        y, z = rt.linear(x.cuda(), w[0].cuda(), b[0].cuda(), **how)
    assert y.dtype == torch.float32 and z.dtype == torch.bfloat16 and bool((base[:, o:] == 7).all())
    inside = torch.zeros(n, dtype=torch.bool)
    for a, e in ranges:
        inside[a:e] = True
    assert bool((base[:, :o].cpu()[~inside] == 7).all())
    tz = sum_bound(i) * mag
    ty = 1.13 * tz + 8 * E32 * (yr.abs() + zr.abs() + (r.double().abs() if residual else 0))
    within((y.cpu().double() - yr)[inside], ty[inside], "y")
    within((z.cpu().double() - zr)[inside], (tz + E16 * zr.abs())[inside], "z")


def test_refusals(rt):  # noqa: F811
    from paper_2604_15380_amd import binding as B
    mk = maker(1)
    x, w, r = mk(6, 8).cuda(), mk(4, 8).cuda(), mk(6, 4).cuda()
    with pytest.raises(ValueError):
        rt.linear(x.float(), w.float(), out=r)
    with pytest.raises(ValueError):
        rt.linear(x, w, out=r.double())
    args = dict(precision=2, rows=6, d_in=8, d_out=4, x=x.data_ptr(), ldx=8, w=w.data_ptr(), y=r.data_ptr(), ldy=4)
    for kw in (dict(y_fp32=2), dict(y_fp32=-1), dict(y_fp32=1, residual=r.data_ptr(), ldr=4)):
        with pytest.raises(B.PainnError) as e:
            B.painn_linear(rt.ctx, B.painn_linear_args(**args, **kw))
        assert e.value.status == -1, kw


@pytest.mark.parametrize("adapter", [0, 96])
def test_tuner_energies_are_not_rounded_to_bf16(rt, adapter):  # noqa: F811
    """The readout against 64 bits, from the activations that it reads."""
    hp, W, batch, model, graph, inp, s, tuner = setup(rt, "bf16", adapter)
    b = tuner.batch(s, batch.struct_ptr, batch.dataset_id)
    e, kept = tuner._forward(b, True)
    name, x, _ = kept["layers"][-1]
    w, bias = (tuner.weight[name + k].double() for k in (".w", ".b"))
    want, _, mag = ref.linear(x.double(), w, bias, "none", None, ref.spans(b["offsets"].tolist(), len(x)))
    assert e.dtype == torch.float32
    within(e.double() - want, sum_bound(x.shape[1]) * mag, "atom energies")
    ptr = batch.struct_ptr
    sums = torch.stack([want[a:c].sum() for a, c in zip(ptr[:-1], ptr[1:])])
    size = torch.stack([mag[a:c].sum() for a, c in zip(ptr[:-1], ptr[1:])])
    within(tuner.energies(b) - sums, (sum_bound(x.shape[1]) + 1e-12) * size, "energies")
    tuner.free()
    graph.free()
    model.free()
