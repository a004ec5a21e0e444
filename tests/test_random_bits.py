"""The random bits that stochastic rounding takes (tests/stats_reference.py writes the kernel's out; test_gpu_optimizer.py holds the kernel to them)."""
import numpy as np

import stats_reference as ref


def test_the_random_bits_are_spread():
    """Of 2^20 entries' bits: each of 256 values of the upper byte as often as the others (chi-square, 255 degrees: mean 255, deviation 22.6), for
    all three uses; neighbours, steps and tensors uncorrelated (six deviations of 2^-10)."""
    draws = {key: ref.random_bits(*key, 1 << 20) for key in [(1, 1, 0), (1, 2, 0), (1, 1, 1), (2, 1, 0)]}
    for parts in draws.values():
        for part in parts:
            counts = np.bincount((part >> np.uint64(8)).astype(np.int64), minlength=256)
            chi = float(((counts - 4096.0) ** 2 / 4096.0).sum())
            assert abs(chi - 255) < 6 * 22.6, chi
    flat = [d.astype(np.float64) / 65536 - 0.5 for parts in draws.values() for d in parts]
    flat += [np.roll(flat[0], s) for s in (1, 2, 64, 256)]
    corr = np.corrcoef(np.stack(flat))
    assert np.abs(corr - np.eye(len(flat))).max() < 6 * 2.0 ** -10
