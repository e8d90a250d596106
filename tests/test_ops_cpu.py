"""CPU checks of the head-tuning operators' boundary: null contexts and
handles give their status without a device, and the packed argument structs
are laid out as the ctypes ones."""
import ctypes
import os

import numpy as np
import pytest

from paper_2604_15380_amd import binding

built = pytest.mark.skipif(not os.path.exists(binding.lib_path()), reason="library not built")


@built
def test_null_contexts_and_handles():
    lib = binding.load_library()
    out, steps = ctypes.c_void_p(), ctypes.c_int64()
    E_ARG = -1
    assert lib.painn_layer_norm(None, 1, 1, 1, None, 1, None, None, 1e-5, None, 1, None, None) == E_ARG
    assert lib.painn_layer_norm_backward(None, 1, 1, 1, None, 1, None, 1, None, None, None, None, 1, None, None) == E_ARG
    for fn in (lib.painn_linear, lib.painn_linear_backward):
        assert fn(None, None) == E_ARG
    for fn in (lib.painn_grouped_linear, lib.painn_grouped_linear_backward):
        assert fn(None, None, 1, None) == E_ARG
    assert lib.painn_adamw_create(None, 0, None, None, ctypes.byref(out)) == E_ARG
    assert lib.painn_adamw_step(None, 1e-3) == E_ARG
    assert lib.painn_adamw_steps(None, ctypes.byref(steps)) == E_ARG
    assert lib.painn_adamw_free(None) == 0


@pytest.mark.parametrize("pack,cls", [(binding.linear_args, binding.painn_linear_args),
                                      (binding.linear_backward_args, binding.painn_linear_backward_args)])
def test_packed_structs(pack, cls):
    values = list(range(3, 3 + len(cls._fields_)))
    got = cls.from_buffer_copy(pack(*values))
    assert [getattr(got, name) for name, _ in cls._fields_] == values


def test_dataset_order():
    from paper_2604_15380_amd.tuning import dataset_order
    ids = np.array([2, 0, 2, 1, 0])
    assert dataset_order(ids).tolist() == [1, 4, 3, 0, 2]
