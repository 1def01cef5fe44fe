"""Gradients as autograd hands them to the norm: parts of larger ones, which start anywhere, views that negate, one number spread out."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _leaves(dtype):
    g = torch.Generator().manual_seed(3)
    return [torch.randn(*s, generator=g).to(dtype).cuda().requires_grad_() for s in ((5, 64), (64,), (5, 64))]


def _grads(loss, leaves):
    return torch.autograd.grad(loss, leaves)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("lead", [1, 3, 8])
def test_parts_of_a_larger_gradient(lib, lead, dtype):
    from paper_2505_24034_amd.autograd import rms_norm
    x, w, r = leaves = _leaves(dtype)
    front = torch.ones(lead, dtype=dtype, device="cuda")
    scale = torch.linspace(-1, 1, lead + x.numel(), device="cuda").to(dtype)
    h, s = rms_norm(x, w, 1e-5, residual=r)
    got = _grads((torch.cat([front, h.flatten()]) * scale).sum() + (torch.cat([front, s.flatten()]) * scale).sum(), leaves)
    h, s = rms_norm(x, w, 1e-5, residual=r)
    want = torch.autograd.grad([h, s], leaves, [scale[lead:].view(5, 64).clone()] * 2)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_views_that_negate(lib):
    from paper_2505_24034_amd.autograd import rms_norm
    x, w, r = leaves = _leaves(torch.float32)
    a, b = (torch.randn(5, 64, device="cuda") for _ in range(2))
    dense = torch._neg_view(a)
    strided = torch.complex(b, b).conj().imag
    assert dense.is_neg() and dense.is_contiguous() and strided.is_neg()
    h, s = rms_norm(x, w, 1e-5, residual=r)
    got = torch.autograd.grad([h, s], leaves, [dense, strided])
    h, s = rms_norm(x, w, 1e-5, residual=r)
    want = torch.autograd.grad([h, s], leaves, [-a, -b])
    assert all(torch.equal(p, q) for p, q in zip(got, want))


def test_a_gradient_of_one_number_spread_out(lib):
    from paper_2505_24034_amd.autograd import rms_norm
    x, w, r = leaves = _leaves(torch.float32)
    h, s = rms_norm(x, w, 1e-5, residual=r)
    got = _grads(h.sum() + s.sum(), leaves)
    h, s = rms_norm(x, w, 1e-5, residual=r)
    want = torch.autograd.grad([h, s], leaves, [torch.ones_like(h), torch.ones_like(s)])
    assert all(torch.equal(p, q) for p, q in zip(got, want))
