"""The head-tuning operators' workspace is their own: enlarging it leaves alone
what a captured forces graph replays on, and the forces leave alone what a
captured operator replays on."""
import pytest
import torch

import synth
from test_gpu_branch import batch

pytestmark = pytest.mark.gpu


def setting():
    from paper_2604_15380_amd import Runtime
    rt = Runtime(0)
    hp = synth.HyperParams(F=64, K=6, L=2, n_species=6, cutoff=3.0, n_heads=2, shared_dims=[50], branch_dims=[32, 1])
    m = rt.load_model(synth.weight_file_bytes(hp, synth.make_weights(hp, 3)))
    build = lambda n: rt.build_graph(rt.upload_batch(batch(n, 2)), hp.cutoff)  # noqa: E731
    return rt, m, build


def test_a_captured_reverse_pass_and_larger_forces():
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        rt, m, build = setting()
        g = build(9000)
        gen = torch.Generator(device="cuda").manual_seed(1)
        rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
        x, dy, w = rnd(3000, 64), rnd(3000, 80), rnd(80, 64)
        want = [a.clone() for a in rt.linear_backward(dy, x, w, activation="silu", preact=dy)]
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = rt.linear_backward(dy, x, w, activation="silu", preact=dy)
        for _ in range(3):
            rt.forces(m, g, "fp32")
            for a in got:
                a.fill_(float("nan"))
            graph.replay()
            assert all(torch.equal(a, b) for a, b in zip(got, want))
        del graph
        g.free()
        m.free()
        rt.close()


def test_a_larger_reverse_pass_and_captured_forces():
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        rt, m, build = setting()
        g = build(60)
        E, F = (a.clone() for a in rt.forces(m, g, "fp32"))
        e, f = torch.empty_like(E), torch.empty_like(F)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            rt.forces(m, g, "fp32", energies=e, forces=f)
        x, dy, w = (torch.ones(*s, device="cuda") for s in ((200000, 256), (200000, 300), (300, 256)))
        for _ in range(3):
            rt.linear_backward(dy, x, w, activation="silu", preact=dy)
            e.fill_(float("nan"))
            f.fill_(float("nan"))
            graph.replay()
            assert torch.equal(e, E) and torch.equal(f, F)
        del graph
        g.free()
        m.free()
        rt.close()
