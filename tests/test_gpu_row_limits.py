"""Calls of as many rows as they may have."""
import pytest
import torch

pytestmark = pytest.mark.gpu
K = 5


def _rows(N, d):
    """zeros but for the last rows"""
    x = torch.zeros(N, d, dtype=torch.bfloat16, device="cuda")
    x[-K:] = torch.randn(K, d, device="cuda")
    return x, x[-K:].clone()


@pytest.mark.parametrize("rows,cols", [(2 ** 26 - 4, 16), (2 ** 23 + 3, 2064), (2 ** 22 + 1, 4112)])
def test_quantise_rows(lib, rows, cols):
    x, last = _rows(rows, cols)
    q, scale = lib.quantise_rows(x)
    want, want_scale = lib.quantise_rows(last)
    assert torch.equal(q[-K:], want) and torch.equal(scale[-K:], want_scale)
    assert not scale[:-K].any() and not q[:1000].any() and not q[rows // 2:rows // 2 + 1000].any()
    del x, q, scale
    torch.cuda.empty_cache()


def test_rms_norm(lib):
    x, last = _rows(2 ** 26 - 4, 8)
    w = torch.randn(8, device="cuda")
    h, s, rstd = lib.rms_norm(x, w, 0.25, residual=x)
    want = lib.rms_norm(last, w, 0.25, residual=last)
    assert torch.equal(h[-K:], want[0]) and torch.equal(s[-K:], want[1]) and torch.equal(rstd[-K:], want[2])
    assert not h[:-K].any() and (rstd[:-K] == 2).all()
    dx, dw = lib.rms_norm_bwd(h, s, w, rstd, dsum=x)
    assert torch.equal(dx[-K:], lib.rms_norm_bwd(*want[:2], w, want[2], dsum=last)[0]) and not dx[:-K].any()
    n = want[1].double() * want[2].double()[:, None]
    # the other rows add zeros, so a column is a chain of at most five terms and as many products of two roundings
    assert ((dw.double() - (want[0].double() * n).sum(dim=0)).abs() <= 8 * 2.0 ** -24 * (want[0].double() * n).abs().sum(dim=0)).all()


def test_verify_drafts(lib):
    B, V, n = 2 ** 24 // 63, 9, 31
    z = torch.randn(B, n + 1, V, dtype=torch.bfloat16, device="cuda")
    y = z[:, :n] + torch.randn(B, n, V, dtype=torch.bfloat16, device="cuda") / 4
    drafts = y.argmax(dim=2).to(torch.int32)
    u = torch.rand(B, n + 1, device="cuda")
    got = lib.verify_drafts(z, drafts, u, draft_logits=y)
    for part in (slice(0, K), slice(B // 2, B // 2 + K), slice(B - K, B)):
        c = lambda t: t[part].contiguous()  # noqa: E731
        want = lib.verify_drafts(c(z), c(drafts), c(u), draft_logits=c(y))
        assert all(torch.equal(a[part], b) for a, b in zip(got, want))
