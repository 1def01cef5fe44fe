"""First moments in 8 bits over many steps, in blocks whose largest entry stays what it is: gradients that change size and sign.

A moment comes to rest where an update, (1 - b1) (g - m), is half a step of its code at most: 2^-4 of its power of two, 2^-10 of the
block's factor below 2^-6.  In units of the factor the kernel's value is within 12 u of 448 (u = 2^-24), the factor itself comes to rest with
the leading entry, whose distance from its gradient is b1^200 = 2.5e-6 of it at the end of the first 200 steps."""
import numpy as np
import pytest
import torch

from operator_util import BLOCK, e4m3_values, f64

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("b1", [0.9, 0.9375])
def test_first_moments_follow_their_gradients(lib, b1):
    n = 1 << 14
    g = np.random.default_rng(3)
    size = np.exp(g.uniform(np.log(1e-5), np.log(0.9), n))
    lead = np.arange(n) % BLOCK == 0
    p = torch.zeros(n, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    ms, vs = (torch.zeros(n // BLOCK, device="cuda") for _ in range(2))
    step = 0
    for share, steps in ((0.4, 200), (0.2, 150), (-0.2, 150), (1.0, 150), (0.0, 150)):
        grad = 1e-3 * np.where(lead, 1.0, share * size)
        G = torch.from_numpy(grad).float().cuda()
        for _ in range(steps):
            step += 1
            lib.adamw_step([p], [G], [m], [v], 0.0, step, betas=(b1, 0.999), exp_avg_scales=[ms], exp_avg_sq_scales=[vs])
        s = np.repeat(f64(ms), BLOCK)
        assert (np.abs(s / (1e-3 / 448) - 1) <= 3e-6).all()
        q = e4m3_values(m)
        half = np.maximum(2.0 ** (np.floor(np.log2(np.maximum(np.abs(q), 2.0 ** -9))) - 4), 2.0 ** -10)
        off = (1 - b1) * np.abs(f64(G) / s - q)
        assert (off <= half + 448 * 3e-6 * (1 - b1) + 12 * U * 448)[~lead].all(), share
        # what is above 2^-6 in its block and has a gradient of the other sign cannot rest
        assert (q * np.sign(share) > -(2.0 ** -6) * (1 + 1e-9))[~lead].all() or share == 0
    assert not p.any()
