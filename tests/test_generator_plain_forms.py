"""The plain forms that the norm's and the generator's kernels are held to, against what they claim to be."""
import numpy as np
import pytest
import torch

from generator_util import quantise_rows, rms, rms_bwd, verify


@pytest.mark.parametrize("N,d,dsum", [(1, 4, False), (5, 12, True), (3, 40, False)])
def test_norm_gradient_is_that_of_differences_and_of_autograd(N, d, dsum):
    g = np.random.default_rng(N + d)
    s, w, dh = g.standard_normal((N, d)), 1 + 0.3 * g.standard_normal(d), g.standard_normal((N, d))
    ds = g.standard_normal((N, d)) if dsum else None

    def f(s, w):
        return (rms(s, w, 1e-3)[0] * dh).sum() + (0.0 if ds is None else (ds * s).sum())

    dx, dw = rms_bwd(dh, s, w, 1e-3, ds)
    vs, vw, e = g.standard_normal((N, d)), g.standard_normal(d), 1e-5
    # a central difference is off by e^2 of the third derivative and 1e-16 / e of the value
    assert abs((f(s + e * vs, w) - f(s - e * vs, w)) / (2 * e) - (dx * vs).sum()) < 1e-7 * (1 + np.abs(dx).sum())
    assert abs((f(s, w + e * vw) - f(s, w - e * vw)) / (2 * e) - (dw * vw).sum()) < 1e-7 * (1 + np.abs(dw).sum())
    ts, tw = torch.tensor(s, requires_grad=True), torch.tensor(w, requires_grad=True)
    h = ts / (ts.square().mean(1, keepdim=True) + 1e-3).sqrt() * tw
    ((h * torch.tensor(dh)).sum() + (0 if ds is None else (ts * torch.tensor(ds)).sum())).backward()
    assert np.allclose(ts.grad.numpy(), dx, rtol=1e-12, atol=1e-12) and np.allclose(tw.grad.numpy(), dw, rtol=1e-12, atol=1e-12)


def test_int8_rows():
    q, s = quantise_rows(np.array([[1.0, -127.0, 63.5, 64.5], [0, 0, 0, 0], [np.inf, 1, 2, 3], [2.0 ** -101, 0, 0, 0]], dtype=np.float32))
    assert q.tolist() == [[1, -127, 64, 64], [0] * 4, [0] * 4, [0] * 4] and s[0] == 1 and s[1] == 0 and np.isnan(s[2]) and s[3] == 0


@pytest.mark.parametrize("model", [True, False])
def test_verified_tokens_have_the_target_s_distribution(model):
    """the first token of 40000 trials of one draft, whatever the draft's distribution: each frequency within five standard deviations"""
    g = np.random.default_rng(3)
    B, V = 40000, 6
    z, y = g.standard_normal(V) * 1.5, g.standard_normal(V) * 1.5
    p, q = np.exp(z) / np.exp(z).sum(), np.exp(y) / np.exp(y).sum()
    drafts = g.choice(V, size=(B, 1), p=q)
    logits = np.broadcast_to(z, (B, 2, V))
    tokens, accepted, logp = verify(logits, drafts, g.random((B, 2)), np.broadcast_to(y, (B, 1, V)) if model else None)
    freq = np.bincount(tokens[:, 0], minlength=V) / B
    assert (np.abs(freq - p) < 5 * np.sqrt(p * (1 - p) / B)).all()
    assert np.allclose(logp[:, 0], np.log(p[tokens[:, 0]]))
    # accepted with the probability that the two have in common, or with p of the draft
    want = np.minimum(p, q).sum() if model else (p * q).sum()
    assert abs((accepted == 1).mean() - want) < 5 * np.sqrt(want * (1 - want) / B)
