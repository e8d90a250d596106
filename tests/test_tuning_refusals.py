"""What HeadTuner refuses before it makes anything on a device."""
import numpy as np
import pytest
import torch

from paper_2604_15380_amd.runtime import Runtime
from paper_2604_15380_amd.tuning import HeadTuner


@pytest.mark.parametrize("groups", [0, -1, -8, 7, 97])
def test_adapter_groups(groups, monkeypatch):
    """Also 0, which is no other adapter."""
    made = []
    monkeypatch.setattr(Runtime, "adamw", lambda self, *a, **how: made.append(a))
    rt = Runtime.__new__(Runtime)
    rt.device = torch.device("cpu")
    weights = {"head0.0.w": np.zeros((1, 64)), "head0.0.b": np.zeros(1)}
    how = dict(F=64, n_heads=1, n_shared=0, n_branch=1, dtype="fp32")
    with pytest.raises(ValueError, match="groups"):
        HeadTuner(rt, weights, adapter=96, adapter_norm="group", adapter_groups=groups, **how)
    assert not made
    # where they are not used they are not looked at
    assert HeadTuner(rt, weights, adapter=96, adapter_groups=groups, **how).groups == 0
    assert HeadTuner(rt, weights, adapter_norm="group", adapter_groups=groups, **how).groups == 0
    assert HeadTuner(rt, weights, adapter=96, adapter_norm="group", adapter_groups=12, **how).groups == 12
    assert len(made) == 3
