"""Outputs that may lie in place of an input: with its row stride they give the
bits of an output of their own, with another one they are refused (a row would
be overwritten before it is read)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def rt():
    from paper_2604_15380_amd import Runtime
    r = Runtime(0)
    yield r
    r.close()


def rows(src, ld):
    """A copy of src with row stride ld, and the view of the same memory with a
    row stride one larger."""
    n, c = src.shape
    base = torch.zeros(n * (ld + 1), dtype=src.dtype, device="cuda")
    v = base[:n * ld].view(n, ld)[:, :c]
    v.copy_(src)
    return v, base.view(n, ld + 1)[:, :c]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("n,i,o", [(300, 40, 72), (9, 130, 33), (5000, 264, 256)])
def test_in_place(rt, dtype, n, i, o):
    from paper_2604_15380_amd import PainnError
    gen = torch.Generator(device="cuda").manual_seed(n)
    rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda").to(DTYPES[dtype])  # noqa: E731
    x, w, r, dy, xz, gamma = rnd(n, i), rnd(o, i), rnd(n, o), rnd(n, o), rnd(n, i), rnd(i)

    def refused(call):
        with pytest.raises(PainnError) as e:
            call()
        assert e.value.status == -1 and "in place" in str(e.value)

    want, mean, rstd = rt.layer_norm(x, gamma, gamma)
    v, other = rows(x, i + 3)
    refused(lambda: rt.layer_norm(v, gamma, gamma, out=other))
    assert torch.equal(rt.layer_norm(v, gamma, gamma, out=v)[0], want)

    dx, dg, db = rt.layer_norm_backward(xz, x, gamma, mean, rstd)
    v, other = rows(xz, i + 3)
    refused(lambda: rt.layer_norm_backward(v, x, gamma, mean, rstd, dx=other))
    got = rt.layer_norm_backward(v, x, gamma, mean, rstd, dx=v)
    assert all(torch.equal(a, b) for a, b in zip(got, (dx, dg, db)))

    want = rt.linear(x, w, activation="silu", residual=r)
    v, other = rows(r, o + 3)
    refused(lambda: rt.linear(x, w, activation="silu", residual=v, out=other))
    assert torch.equal(rt.linear(x, w, activation="silu", residual=v, out=v), want)

    want = rt.linear_backward(dy, x, w, x_activation="silu", x_preact=xz)
    v, other = rows(xz, i + 3)
    refused(lambda: rt.linear_backward(dy, x, w, x_activation="silu", x_preact=v, dx=other))
    got = rt.linear_backward(dy, x, w, x_activation="silu", x_preact=v, dx=v)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
