"""FP32 wide branches where an infinite activation meets an infinite weight:
the product is an infinity of their signs, as in FP32 arithmetic."""
import numpy as np
import pytest

import synth
from test_gpu_branch import batch, rt  # noqa: F401
from test_gpu_branch_nonfinite import UNIT

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_infinite_activation_and_weight(rt, sign):  # noqa: F811
    hp = synth.HyperParams(F=64, K=6, L=1, n_species=6, cutoff=3.0, n_heads=1, shared_dims=[],
                           branch_dims=[256, 256, 1])
    W = synth.make_weights(hp, 80)
    W["head0.0.w"][UNIT] = 0.0
    W["head0.0.b"][UNIT] = 1e39                       # the activation is +inf on every atom
    W["head0.1.w"][:, UNIT] = 2.0 ** -10              # one plane
    W["head0.1.w"][7, UNIT] = 1e39                    # past FP32's range: an infinity
    W["head0.2.w"][0] = sign * np.abs(W["head0.2.w"][0])
    m = rt.load_model(synth.weight_file_bytes(hp, W))
    b = batch(40, 2)
    b.dataset_id[:] = 0
    g = rt.build_graph(rt.upload_batch(b), hp.cutoff)
    E = rt.forward(m, g, "fp32").cpu().numpy()
    assert np.all(E == sign * np.inf), E
    g.free()
    m.free()
