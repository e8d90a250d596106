"""AdamW and the life of its context: an optimizer left over from a closed
context refuses, can be freed, and leaves the others alone."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_steps_after_the_context_are_refused():
    from paper_2604_15380_amd import PainnError, Runtime
    rt, other = Runtime(0), Runtime(0)
    p = [torch.ones(300, device="cuda") for _ in range(5)]
    g = [torch.full((300,), 0.5, device="cuda") for _ in range(5)]
    opts = [rt.adamw([a], [b], state_bits=bits) for a, b, bits in zip(p[:4], g, (32, 8, 32, 8))]
    alive = other.adamw([p[4]], [g[4]])
    for o in opts + [alive]:
        o.step()
    opts[1].free()                       # from between the others
    opts[3].free()                       # and the newest
    want = [a.clone() for a in p]
    rt.close()
    for o in (opts[0], opts[2]):
        with pytest.raises(PainnError) as e:
            o.step()
        assert e.value.status == -1 and o.steps == 1
        o.free()
        with pytest.raises(PainnError):
            o.step()
        o.free()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(p, want))
    alive.step()
    torch.cuda.synchronize()
    assert alive.steps == 2 and bool((p[4] != want[4]).all())
    alive.free()
    other.close()


def test_a_context_closed_before_its_optimizer_is_collected():
    from paper_2604_15380_amd import Runtime
    rt = Runtime(0)
    o = rt.adamw([torch.ones(10, device="cuda")], [torch.ones(10, device="cuda")])
    o.step()
    rt.close()
    del o
    torch.cuda.synchronize()
