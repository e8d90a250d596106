"""Dense and grouped layers at sizes that fill the GPU, where the larger tiles,
the long contractions and the chunks of the weight gradient are taken, against
the 64-bit form (torch.float64 products on the GPU); bounds as in
test_gpu_dense.py.  And: calls on another stream, calls in a HIP graph."""
import pytest
import torch

import ops_reference as ref
from ops_reference import E16, E32, sum_bound, within

pytestmark = pytest.mark.gpu

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


def maker(seed, dtype):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *s, scale=1.0: (torch.randn(*s, generator=g, device="cuda") * scale).to(dtype)


def ragged(n, groups):
    """Offsets of groups whose sizes differ widely, some of them empty."""
    cuts = [0] + [int(n * ((k + 1) / groups) ** 2.5) for k in range(groups)]
    cuts[3] = cuts[4]
    cuts[-1] = n
    return cuts


# rows, d_in, d_out, groups: 256 x 256 tiles, 128 x 160, 128 x 128; strides that
# are no multiple of 16 bytes; one wide and one narrow contraction
CASES = [("bf16", 70000, 256, 1024, 0), ("bf16", 66000, 776, 776, 0), ("bf16", 66000, 776, 776, 16),
         ("bf16", 40001, 1024, 1024, 5), ("bf16", 30000, 256, 384, 0), ("bf16", 30000, 337, 776, 16),
         ("bf16", 3000, 4096, 520, 0), ("bf16", 9000, 50, 776, 70), ("bf16", 65536, 64, 1, 0),
         ("fp32", 20000, 337, 776, 0), ("fp32", 20000, 776, 776, 16), ("fp32", 1500, 4100, 300, 0)]


@pytest.mark.parametrize("dtype,n,i,o,groups", CASES)
def test_forward_and_backward(rt, dtype, n, i, o, groups):
    t = DTYPES[dtype]
    mk = maker(n + i, t)
    G = groups or 1
    cuts = ragged(n, groups) if groups else [0, n]
    ranges = ref.spans(cuts, n)
    off = torch.tensor(cuts, dtype=torch.int32, device="cuda")
    x, w, b, r = mk(n, i), mk(G, o, i, scale=i ** -0.5), mk(G, o), mk(n, o)
    half = E16 if dtype == "bf16" else 0.0

    how = dict(activation="silu", residual=r, keep_preact=True)
    y, z = rt.grouped_linear(x, w, off, b, **how) if groups else rt.linear(x, w[0], b[0], **how)
    yr, zr, mag = ref.linear(x.double(), w.double(), b.double(), "silu", r.double(), ranges)
    tz = sum_bound(i) * mag
    within(z.double() - zr, tz + half * zr.abs(), "z")
    within(y.double() - yr, 1.13 * tz + 8 * E32 * (yr.abs() + zr.abs() + r.double().abs()) + half * yr.abs(), "y")
    del yr, zr, mag, tz, y

    dy, xz = mk(n, o), mk(n, i, scale=2.0)
    how = dict(activation="silu", preact=z, x_activation="silu", x_preact=xz)
    back = (lambda: rt.grouped_linear_backward(dy, x, w, off, **how)) if groups else \
           (lambda: rt.linear_backward(dy, x, w[0], **how))
    dx, dw, db = back()
    e = ref.linear_backward(dy.double(), z.double(), "silu", x.double(), w.double(), xz.double(), "silu", ranges)
    dw, db = (dw, db) if groups else (dw[None], db[None])
    rows = max(c - a for a, c in ranges)
    for name, mine, k in (("dx", dx, o), ("dw", dw, rows), ("db", db, rows)):
        within(mine.double() - e[name], (sum_bound(k) + half) * e["m" + name] + 16 * E32 * e["e" + name]
               + half * e[name].abs(), name)
    again = back()
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1] if groups else again[1][None])
    assert torch.equal(db, again[2] if groups else again[2][None])


def test_another_stream(rt):
    """Inputs made and outputs used on a stream that is not the context's: the
    bits of the same calls on the context's stream."""
    gen = torch.Generator(device="cuda").manual_seed(11)
    w = torch.randn(300, 200, device="cuda", generator=gen)
    ones, zeros = torch.ones(300, device="cuda"), torch.zeros(300, device="cuda")
    base = torch.randn(4000, 200, device="cuda", generator=gen)
    want = []
    for k in range(20):
        y = rt.linear(base * float(k), w)
        n, mean, rstd = rt.layer_norm(y, ones, zeros)
        want.append((y.clone(), n.clone(), mean.clone(), rstd.clone()))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for k in range(20):
            x = base * float(k)
            y = rt.linear(x, w)
            n, mean, rstd = rt.layer_norm(y, ones, zeros)
            got = [a + 0.0 for a in (y, n, mean, rstd)]
            del x, y, n, mean, rstd
            assert all(torch.equal(a, b) for a, b in zip(got, want[k])), k
    torch.cuda.synchronize()


def test_in_a_graph():
    """Forward, reverse and an optimizer step captured once, replayed on new
    inputs with eager work between, each replay against eager calls."""
    from paper_2604_15380_amd import Runtime
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        rt = Runtime(0)
        gen = torch.Generator(device="cuda").manual_seed(3)
        rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()  # noqa: E731
        n, i, o, G = 3000, 72, 136, 3
        x, dy, w, b = rnd(n, i), rnd(n, o), rnd(G, o, i), rnd(G, o)
        off = torch.tensor([0, 700, 700, n], dtype=torch.int32, device="cuda")
        gamma, beta = rnd(i), rnd(i)
        master = w.float()
        out = {}

        def work():
            h, mean, rstd = rt.layer_norm(x, gamma, beta)
            y, z = rt.grouped_linear(h, w, off, b, activation="silu", keep_preact=True)
            dh, dw, db = rt.grouped_linear_backward(dy, h, w, off, activation="silu", preact=z)
            dx, dg, dbeta = rt.layer_norm_backward(dh, x, gamma, mean, rstd)
            return dict(y=y, dw=dw, db=db, dx=dx, dg=dg, dbeta=dbeta)

        eager = work()          # (also makes the workspace)
        grad = torch.zeros_like(w)
        opt = rt.adamw([master], [grad], copies=[w])
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = work()
            grad.copy_(out["dw"])
            opt.step()
        for k in range(4):
            x.copy_(rnd(n, i))
            dy.copy_(rnd(n, o))
            before, w0 = master.clone(), w.clone()
            state = [a.clone() for a in opt.m + opt.v]
            graph.replay()
            stream.synchronize()
            got = {key: a.clone() for key, a in out.items()}
            after = master.clone()
            w.copy_(w0)
            eager = work()
            stream.synchronize()
            for key in eager:
                assert torch.equal(got[key], eager[key]), (k, key)
            check = rt.adamw([before], [eager["dw"]], copies=[w], steps=opt.steps - 1,
                             state=dict(m=state[:1], v=state[1:]))
            check.step()
            stream.synchronize()
            assert torch.equal(after, before)
            torch.randn(1000, device="cuda").sum().item()
        opt.free()
        rt.close()


def test_a_workspace_under_capture_is_refused():
    from paper_2604_15380_amd import PainnError, Runtime
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        rt = Runtime(0)
        x, dy, w = (torch.randn(*s, device="cuda") for s in ((5000, 64), (5000, 80), (80, 64)))
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            with pytest.raises(PainnError) as e:
                rt.linear_backward(dy, x, w)
            keep = x + 1.0
        assert e.value.status == -2 and "captur" in str(e.value)
        graph.replay()
        assert torch.equal(keep, x + 1.0)
        rt.linear_backward(dy, x, w)
        stream.synchronize()
        rt.close()
