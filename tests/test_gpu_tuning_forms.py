"""HeadTuner's boundary: what it takes for reference energies."""
import pytest
import torch

from test_gpu_tuning import rt, setup  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [lambda n: (n, 1), lambda n: (1, n), lambda n: (1,), lambda n: (n + 1,)])
def test_reference_energies_of_another_shape(rt, shape):  # noqa: F811
    """[n, 1] would be compared with every structure's energy ([n, n])."""
    hp, W, batch, model, graph, inp, s, tuner = setup(rt, "fp32", 0)
    b = tuner.batch(s, batch.struct_ptr, batch.dataset_id)
    before = {k: v.clone() for k, v in tuner.master.items()}
    with pytest.raises(ValueError):
        tuner.step(b, torch.zeros(shape(batch.n_struct), dtype=torch.float64, device="cuda"))
    assert tuner.optimizer.steps == 0 and all(torch.equal(v, before[k]) for k, v in tuner.master.items())
    zeros = torch.zeros(batch.n_struct, dtype=torch.float64, device="cuda")
    assert float(tuner.gradients(b, 0.0)) == float(tuner.gradients(b, zeros)) > 0
    tuner.free()
    graph.free()
    model.free()
