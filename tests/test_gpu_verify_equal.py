"""Drafts whose logits are the target's plus a constant: p and q are one distribution, whatever the powers of either are off by, and the token behind a
draft that is refused all the same (it lies outside the vocabulary) comes out of p.

A power is off by at most 1.06e-12 of itself.  An entry of p is a power, times the row's scale, over a sum of powers times their chunk's two scales: five of them,
so p - q leaves at most ten, 1.06e-11, and sums of up to 2^21 terms in 64 bits another 1e-13 at most: less than the 2^-36 = 1.46e-11 from which on it is drawn from."""
import numpy as np
import pytest
import torch

from test_gpu_verify import _check, _run

pytestmark = pytest.mark.gpu


def _shifted(B, V, seed, whole):
    """logits that are multiples of 1/64 and so exact with any of the constants; without `whole` one to three of each 8192, and nothing else"""
    g = np.random.default_rng(seed)
    z = np.full((B, 2, V), -np.inf, dtype=np.float32)
    if whole:
        z[:] = g.integers(-256, 256, (B, 2, V)) / 64
    else:
        for first in range(0, V, 8192):
            size = min(8192, V - first)
            for _ in range(3):
                z[np.arange(B), 0, first + g.integers(0, size, B)] = g.integers(-128, 128, B) / 64
        z[:, 1] = 0.0
    y = (z[:, :1] + (g.integers(-6 * 64, 6 * 64, (B, 1, 1)) / 64).astype(np.float32)).astype(np.float32)
    return z, y, g.random((B, 2)).astype(np.float32) * np.float32(1 - 2.0 ** -23), (0.3 + 1.7 * g.random(B)).astype(np.float32)


@pytest.mark.parametrize("whole", [False, True])
@pytest.mark.parametrize("B,V", [(300, 40), (300, 8192), (300, 3 * 8192), (300, 40000)])
def test_drafts_with_the_target_s_distribution(lib, B, V, whole):
    z, y, u, temps = _shifted(B, V, V, whole)
    x = torch.from_numpy(z), torch.from_numpy(y), np.full((B, 1), -1, dtype=np.int32), u, None, temps
    got = _run(lib, *x)
    assert not got[1].any()
    _check(got, *x)
