"""First moments in 8 bits are rounded to nearest: which rates of decay they can follow.  No kernel runs."""
import ctypes

import numpy as np
import pytest
import torch

from operator_util import E4M3, e4m3_nearest
from paper_2505_24034_amd import binding as L
from paper_2505_24034_amd.optim import AdamW

no_gpu_only = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="fake device pointers: CPU-only test")


def _followed(b1, g, steps=400):
    """m of an entry, in units of its block's factor, that starts at every code above 2^-6 and sees the gradient g * m from then on"""
    m = E4M3[E4M3 > 2.0 ** -6]
    g = g * m
    for _ in range(steps):
        m = e4m3_nearest(np.clip(b1 * m + (1 - b1) * g, -448, 448))
    return m, g


def test_the_largest_rate_that_leaves_no_moment_where_it_was():
    normal = E4M3[E4M3 > 2.0 ** -6]                                        # at that one the steps below are as wide as those above
    for b1 in (0.5, 0.9, L.STATE_BETA1):
        assert (e4m3_nearest(b1 * normal) < normal).all()                  # a gradient of zero takes every one down
        m, g = _followed(b1, -0.5)
        assert (m[normal >= 1] < 0).all()                                  # and one of the other sign turns it
        m, g = _followed(b1, 0.5)
        half = np.maximum(2.0 ** (np.floor(np.log2(m)) - 4), 2.0 ** -10)
        assert ((1 - b1) * np.abs(g - m) <= half).all()
    for b1 in (0.95, 0.98):
        assert (e4m3_nearest(b1 * normal) == normal).any()
    m, _ = _followed(0.98, -0.5)
    assert (m > 0).any()                                                   # stands still on the wrong side


@no_gpu_only
@pytest.mark.parametrize("beta1,ok", [(0.9375, True), (0.94, False), (0.95, False), (0.99, False)])
def test_larger_ones_are_refused(beta1, ok):
    lib = L.load()
    p = L.AdamwParams(lr=1e-3, beta1=beta1, beta2=0.999, eps=1e-8, weight_decay=0.0, step=1)

    def status(n, bits8):
        at = 1 << 24
        full = L.AdamwTensor(param=at, grad=at + 4096, m=at + 8192, v=at + 12288, m_scale=at + 16384 if bits8 else None,
                             v_scale=at + 20480 if bits8 else None, n=n, param_dt=L.F32, grad_dt=L.F32)
        # behind it one that is refused for another reason: nothing is launched here
        bad = L.AdamwTensor(param=None, n=1, param_dt=L.F32, grad_dt=L.F32)
        code = lib.llamarl_adamw_step((L.AdamwTensor * 2)(full, bad), 2, ctypes.byref(p), None, None, None, None)
        assert code == L.ERR_INVALID_ARG
        return b"beta1" in lib.llamarl_last_error()

    assert status(100, True) == (not ok)
    assert not status(100, False) and not status(0, True)


def test_the_optimiser_refuses_them_before_anything_moves(monkeypatch):
    calls = []
    monkeypatch.setattr(L, "adamw_step", lambda *a, **kw: calls.append(a))
    p = [torch.nn.Parameter(torch.zeros(4)) for _ in range(2)]
    with pytest.raises(L.LlamarlError, match="betas"):
        AdamW(p, betas=(0.95, 0.999), state_bits=8)
    with pytest.raises(L.LlamarlError, match="betas"):
        AdamW([dict(params=p[:1]), dict(params=p[1:], betas=(0.99, 0.9))], state_bits=8)
    AdamW(p, betas=(0.99, 0.999))
    opt = AdamW([dict(params=p[:1]), dict(params=p[1:])], betas=(0.9375, 0.999), state_bits=8)
    for x in p:
        x.grad = torch.ones(4)
    opt.param_groups[1]["betas"] = (0.95, 0.999)                           # as a schedule of momentum sets them
    with pytest.raises(L.LlamarlError, match="betas"):
        opt.step()
    assert not calls and not any("step" in s for s in opt.state.values())
    opt.param_groups[1]["betas"] = (0.85, 0.999)
    opt.step()
    assert len(calls) == 2
    saved = AdamW([dict(params=p[:1]), dict(params=p[1:])], betas=(0.95, 0.999)).state_dict()
    with pytest.raises(L.LlamarlError, match="betas"):
        opt.load_state_dict(saved)
