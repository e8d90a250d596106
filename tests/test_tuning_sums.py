"""HeadTuner's structure energies: each structure's atoms are added by
themselves, so that neither a value that is not finite nor the size of the
other structures' energies reaches them, and always in the same order.

A sum of n values in FP64 by at most ceil(log64 n) levels of 64 is within
64 ceil(log64 n) roundings of the sum of the magnitudes."""
import math
from types import SimpleNamespace

import numpy as np
import pytest
import torch

DEVICES = ["cpu", pytest.param("cuda", marks=pytest.mark.gpu)]
SIZES = [3, 0, 1, 2, 63, 64, 65, 0, 200, 4096, 4097, 9000, 1, 70000, 5, 0]


def tuner_on(device):
    from paper_2604_15380_amd.tuning import HeadTuner
    t = HeadTuner.__new__(HeadTuner)
    t.rt, t.F, t.n_heads, t.dtype = SimpleNamespace(device=torch.device(device)), 2, 4, torch.float32
    return t


def batch(device, sizes):
    t = tuner_on(device)
    ptr = np.concatenate([[0], np.cumsum(sizes)])
    b = t.batch(torch.zeros(int(ptr[-1]), 2, device=device), ptr, np.sort(np.arange(len(sizes)) % 4))
    return t, ptr, b


def sums(t, b, e):
    return t._sum(b, torch.as_tensor(e, device=b["s"].device).view(-1, 1)).cpu().numpy()


@pytest.mark.parametrize("device", DEVICES)
@pytest.mark.parametrize("sizes", [SIZES, [1], [0], [0, 0, 7], [65] * 30, [2] * 500])
def test_sums_and_their_bits(device, sizes):
    t, ptr, b = batch(device, sizes)
    rng = np.random.default_rng(len(sizes))
    e = rng.standard_normal(int(ptr[-1])).astype(np.float32)
    got = sums(t, b, e)
    assert got.shape == (len(sizes),) and got.dtype == np.float64
    for k, n in enumerate(sizes):
        own = e[ptr[k]:ptr[k + 1]].astype(np.float64)
        levels = max(1, math.ceil(math.log(max(n, 2), 64)))
        assert abs(got[k] - math.fsum(own)) <= 64 * levels * 2.0 ** -53 * math.fsum(np.abs(own)), (k, n)
    for _ in range(20):
        assert np.array_equal(sums(t, b, e), got)


@pytest.mark.parametrize("device", DEVICES)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_bad_atom_stays_in_its_structure(device, bad):
    t, ptr, b = batch(device, SIZES)
    e = np.random.default_rng(1).standard_normal(int(ptr[-1])).astype(np.float32)
    clean = sums(t, b, e)
    k = SIZES.index(200)
    e[ptr[k] + 150] = bad
    got = sums(t, b, e)
    rest = np.arange(len(SIZES)) != k
    assert np.array_equal(got[rest], clean[rest]) and np.isfinite(clean).all()
    assert np.isnan(got[k]) if np.isnan(bad) else got[k] == bad


@pytest.mark.parametrize("device", DEVICES)
def test_a_small_structure_beside_large_ones(device):
    """One atom of 2^-20 behind 70,000 of 2^20 keeps all its digits."""
    sizes = [70000, 1, 3]
    t, ptr, b = batch(device, sizes)
    e = np.full(int(ptr[-1]), 2.0 ** 20, dtype=np.float32)
    e[70000:] = np.float32(1 + 2.0 ** -23) * np.float32(2.0 ** -20)
    got = sums(t, b, e)
    assert got[0] == 70000 * 2.0 ** 20 and got[1] == float(e[70000]) and got[2] == 3 * float(e[70000])
