"""BF16 grouped layers whose tiles are 256 x 256, with ragged and empty groups,
against the 64-bit form (the check of test_gpu_dense_large.py).

The tiles by the cost rule: 65,502 x 1,024 -> 1,024 with 16 groups takes 256 x
256 forward and in dx; 33,000 x 1,000 -> 256 forward, with a width that ends
inside a tile's k-block; 20,000 x 512 -> 1,016 in dx; 65,502 x 264 -> 1,000
forward, 128 x 160 in dx.  test_gpu_dense_large.py's grouped cases take 128 x 128
and 128 x 160, its ungrouped ones 256 x 256."""
import pytest

import test_gpu_dense_large as large
from test_gpu_dense_large import rt  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,i,o,groups", [(65502, 1024, 1024, 16), (33000, 1000, 256, 7), (20000, 512, 1016, 4),
                                          (65502, 264, 1000, 16)])
def test_tiles_of_256(rt, n, i, o, groups):  # noqa: F811
    large.test_forward_and_backward(rt, "bf16", n, i, o, groups)
