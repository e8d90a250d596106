"""CPU checks of group norm, the gate and the gradient norm: null contexts and
handles, the packed structs, the workspaces' sizes, and what Runtime refuses
before it calls the library."""
import ctypes
import os

import pytest
import torch

from paper_2604_15380_amd import binding
from paper_2604_15380_amd.runtime import AdamW, Gate, GradNorm, Runtime

built = pytest.mark.skipif(not os.path.exists(binding.lib_path()), reason="library not built")


@built
def test_null_contexts_and_handles():
    lib = binding.load_library()
    out = ctypes.c_void_p()
    E_ARG = -1
    assert lib.painn_group_norm(None, None) == E_ARG
    assert lib.painn_group_norm_backward(None, None, None, 1, None, 1, None, None) == E_ARG
    assert lib.painn_gate(None, None) == E_ARG
    assert lib.painn_gate_backward(None, None, None, 0.0, None, 1) == E_ARG
    assert lib.painn_grad_norm_create(None, 0, None, ctypes.byref(out)) == E_ARG
    assert lib.painn_grad_norm_compute(None, 1.0, None) == E_ARG
    assert lib.painn_grad_norm_clip(None, 1.0, None) == E_ARG
    assert lib.painn_grad_norm_free(None) == 0
    assert lib.painn_adamw_step_scaled(None, 1e-3, None) == E_ARG


@pytest.mark.parametrize("pack,cls", [(binding.group_norm_args, binding.painn_group_norm_args),
                                      (binding.gate_args, binding.painn_gate_args)])
def test_packed_structs(pack, cls):
    values = [float(i) if t is ctypes.c_double else i for i, (_, t) in enumerate(cls._fields_, 3)]
    got = cls.from_buffer_copy(pack(*values))
    assert [getattr(got, name) for name, _ in cls._fields_] == values


@built
def test_workspace_sizes():
    """None where every sample fits a team; sums of tiles where one may be
    longer; bounded whatever the rows."""
    size = binding.painn_group_norm_workspace
    assert size(1, 96, 337, 1, 1, 0, 0, False) == 0
    assert size(1, 65502, 256, 16, 1871, 0, 250, False) == 0
    assert size(1, 65502, 256, 16, 1871, 0, 0, False) > 0
    assert size(1, 147456, 256, 32, 144, 1024, 0, False) == 0
    for rows in (1, 100, 10_000, 10_000_000, 2**31 - 1):
        for cols, groups in ((1, 1), (256, 16), (1000, 1), (64, 64)):
            for samples in (1, 3, 1000):
                for prec in (1, 2):
                    fwd, back = (size(prec, rows, cols, groups, samples, 0, 0, b) for b in (False, True))
                    assert 0 <= fwd <= 513 * 2 * groups * 16 + 256
                    assert fwd <= back <= fwd + 256 + (2048 + 513) * 2 * cols * 4
    assert size(0, 10, 4, 2, 1, 0, 0, False) == 0 and size(1, 10, 4, 3, 1, 0, 0, False) == 0
    gate = binding.painn_gate_workspace
    assert gate(1, 200, 16, 2) == 0 and gate(2, 0, 16, 2) == 0
    for rows in (10**5, 2**31 - 1):
        assert 0 < gate(1, rows, 64, 2) <= 512 * (64 + 65) * 4 + 512


def runtime():
    rt = Runtime.__new__(Runtime)           # no device: only what is checked before it
    rt.device, rt.ctx = torch.device("cpu"), 0
    return rt


def test_group_norm_arguments():
    rt = runtime()
    x, g, off = torch.ones(6, 12), torch.ones(12), torch.tensor([0, 6], dtype=torch.int32)
    stat = torch.ones(1, 3)
    bad = [dict(groups=5), dict(groups=0), dict(groups=24), dict(x=x.double()), dict(x=x[0]), dict(x=x.t()),
           dict(weight=g[:11]), dict(bias=g.bfloat16()), dict(offsets=None), dict(sample_rows=3), dict(activation="tanh"),
           dict(offsets=off.long()), dict(offsets=off[:0]), dict(offsets=off.view(1, 2)),
           dict(offsets=None, sample_rows=4), dict(offsets=None, sample_rows=0), dict(out=torch.ones(6, 13)),
           dict(out=x.bfloat16())]
    for change in bad:
        with pytest.raises(ValueError):
            rt.group_norm(**{**dict(x=x, weight=g, bias=g, groups=3, offsets=off), **change})
    bad = [c for c in bad if "out" not in c] + [dict(mean=torch.ones(1, 4)), dict(rstd=stat.double()), dict(dy=x[:5]),
                                                dict(dx=x[:, :11]), dict(dweight=g[:3]), dict(dbias=g.bfloat16())]
    for change in bad:
        with pytest.raises(ValueError):
            rt.group_norm_backward(**{**dict(dy=x, x=x, weight=g, bias=g, mean=stat, rstd=stat, groups=3, offsets=off),
                                      **change})


def test_gate_arguments():
    rt = runtime()
    x = torch.ones(6, 12)
    for change in (dict(k=0), dict(k=13), dict(logits=x.half()), dict(logits=x[0]), dict(logits=x.t())):
        with pytest.raises(ValueError):
            rt.gate(**{**dict(logits=x, k=2), **change})
    gate = Gate(torch.ones(6, 2), torch.zeros(6, 2, dtype=torch.int32), None, None, None,
                torch.zeros(13, dtype=torch.int32), False)
    dw = torch.ones(6, 2)
    for change in (dict(dweights=dw[:5]), dict(dweights=dw.double()), dict(logits=x[:5]), dict(dlogits=x.bfloat16()),
                   dict(gate=gate._replace(totals=gate.totals[:12])), dict(gate=gate._replace(indices=gate.indices.long()))):
        with pytest.raises(ValueError):
            rt.gate_backward(**{**dict(dweights=dw, logits=x, gate=gate), **change})


def test_grad_norm_arguments():
    rt, a = runtime(), torch.ones(10)
    for grads, outs in (([a], []), ([a.half()], None), ([a[::2]], None), ([a], [a[:9]]), ([a], [a.bfloat16()])):
        with pytest.raises(ValueError):
            GradNorm(rt, grads, outs)
    opt = AdamW.__new__(AdamW)
    opt.rt, opt.handle = rt, 0
    for scale in (torch.ones(2), torch.ones(1, dtype=torch.float64)):
        with pytest.raises(ValueError):
            opt.step(grad_scale=scale)
