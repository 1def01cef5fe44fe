"""The norm in front of the head against its definition in 64 bits.

u = 2^-24 is half a step of fp32.  h is three roundings of its exact value (rstd, and two products), and one of its type.  A dot product of d
terms is a chain of at most 32 in a thread, six steps of a wavefront and 16 of a workgroup: 64 u of the sum of magnitudes covers it.  A column
of dw is a chain over the rows of a workgroup, of the workgroups of a slice and of slices: fewer additions than there are rows, and 80."""
import numpy as np
import pytest
import torch

from generator_util import HALF, U, rms, rms_bwd
from operator_util import f64

pytestmark = pytest.mark.gpu
EPS = 1e-5
SHAPES = [(1, 8), (4, 16), (5, 520), (3, 1032), (2, 1544), (7, 2048), (3, 2056), (1, 4096), (2, 5000), (5, 8192), (2, 8200), (3, 16384),
          (333, 528), (512, 1032), (513, 1032), (1100, 520), (600, 2056), (520, 4104), (514, 8208), (4100, 64)]


def _rows(N, d, dtype, seed, w_dtype=None):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    size = torch.exp(0.7 * r(1, d))
    return ((r(N, d) * size).to(dtype).cuda(), (r(N, d) * size).to(dtype).cuda(), (1 + 0.3 * r(d)).to(w_dtype or dtype).cuda(),
            r(N, d).to(dtype).cuda(), r(N, d).to(dtype).cuda())


def _check_forward(x, residual, w, h, s, rstd, eps=EPS):
    want_s = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    assert torch.equal(s, want_s)
    want, _, r = rms(f64(s), f64(w), eps)
    assert (np.abs(f64(rstd) / r[:, 0] - 1) <= 1.01 * U).all()
    assert (np.abs(f64(h) - want) <= (4 * U + (0 if h.dtype == torch.float32 else HALF[str(h.dtype)])) * np.abs(want)).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,d", SHAPES)
def test_forward_and_backward(lib, N, d, dtype):
    for i, residual in enumerate((True, False)):
        x, res, w, dh, dsum = _rows(N, d, dtype, N + d + i, torch.float32 if (N + i) % 2 else torch.bfloat16)
        res, dsum = (res, dsum) if residual else (None, None)
        h, s, rstd = lib.rms_norm(x, w, EPS, residual=res)
        _check_forward(x, res, w, h, s, rstd)
        dx, dw = lib.rms_norm_bwd(dh, s, w, rstd, dsum=dsum)
        assert dx.dtype == dtype and dw.dtype == w.dtype
        ws, g = f64(w), f64(dh) * f64(w)
        want, want_dw = rms_bwd(f64(dh), f64(s), ws, EPS, None if dsum is None else f64(dsum))
        _, n, r = rms(f64(s), ws, EPS)
        own = r * (8 * U * np.abs(g) + np.abs(n) * 72 * U * np.abs(g * n).mean(axis=1, keepdims=True))
        last = (HALF[str(dtype)] if dtype != torch.float32 else 0) + 3 * U
        assert (np.abs(f64(dx) - want) <= own * 1.01 + last * np.abs(want) + (0 if dsum is None else 3 * U * np.abs(f64(dsum)))).all()
        half = HALF[str(w.dtype)] if w.dtype != torch.float32 else 0
        assert (np.abs(f64(dw) - want_dw) <= (N + 84) * U * np.abs(f64(dh) * n).sum(axis=0) * (1 + half) + (half + U) * np.abs(want_dw)).all()
        again = lib.rms_norm_bwd(dh, s, w, rstd, dsum=dsum)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


@pytest.mark.parametrize("N,d", [(1, 4), (3, 516), (5, 1028), (2, 4100), (9, 260), (700, 1028), (530, 4100), (520, 12)])
def test_fp32_rows_of_four(lib, N, d):
    x, res, w, dh, _ = _rows(N, d, torch.float32, d, torch.bfloat16 if N % 2 else torch.float32)
    h, s, rstd = lib.rms_norm(x, w, EPS, residual=res)
    _check_forward(x, res, w, h, s, rstd)
    dx, dw = lib.rms_norm_bwd(dh, s, w, rstd, dweight_dtype=torch.float32)
    want, want_dw = rms_bwd(f64(dh), f64(s), f64(w), EPS)
    _, n, r = rms(f64(s), f64(w), EPS)
    g = f64(dh) * f64(w)
    assert (np.abs(f64(dx) - want) <= r * (8 * U * np.abs(g) + np.abs(n) * 72 * U * np.abs(g * n).mean(axis=1, keepdims=True)) + 4 * U * np.abs(want)).all()
    assert dw.dtype == torch.float32 and (np.abs(f64(dw) - want_dw) <= (N + 84) * U * np.abs(f64(dh) * n).sum(axis=0)).all()
    only, none = lib.rms_norm_bwd(dh, s, w, rstd, want_dweight=False)
    assert none is None and torch.equal(only, dx)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,d", [(1, 16), (5, 528), (3, 1040), (2, 2048), (7, 4096), (2, 8208), (1, 16384), (300, 272), (65, 4112)])
def test_outputs_in_8_bits_are_those_of_the_quantisers(lib, N, d, dtype):
    x, res, w, _, _ = _rows(N, d, dtype, 3 * N + d)
    q, scale, s = lib.rms_norm_rows(x, w, EPS, residual=res)
    qb, scale_b, s_b = lib.rms_norm_blocks(x, w, EPS, residual=res)
    h, _, _ = lib.rms_norm(s.float(), w.float(), EPS)                      # the same numbers in fp32
    want, want_scale = lib.quantise_rows(h)
    assert torch.equal(q, want) and torch.equal(scale, want_scale) and torch.equal(s, s_b)
    want, want_scale = lib.quantise_blocks(h, 1)
    assert torch.equal(qb.view(torch.uint8), want.view(torch.uint8)) and torch.equal(scale_b.view(torch.uint8), want_scale.view(torch.uint8))
    # and int8 by its definition: scale and quotient are a few roundings from exact, 127 steps the largest
    exact = rms(f64(s), f64(w), EPS)[0]
    top = np.abs(exact).max(axis=1)
    assert (np.abs(f64(scale) * 127 / top - 1) <= 6 * U).all()
    assert (np.abs(f64(q) - exact / (top / 127)[:, None]) <= 0.5 + 127 * 12 * U).all()


@pytest.mark.parametrize("size", [1e30, 3e37, 1e-30, 1e-18])
def test_squares_beyond_fp32(lib, size):
    x, _, w, _, _ = _rows(4, 520, torch.float32, 9)
    x *= size / float(x.abs().max())
    eps = 1e-36 if size < 1 else EPS
    h, s, rstd = lib.rms_norm(x, w, eps)
    _check_forward(x, None, w, h, s, rstd, eps=float(np.float32(eps)))


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("d", [528, 4096])
def test_a_row_that_is_not_finite_keeps_to_itself(lib, value, d):
    x, res, w, dh, _ = _rows(9, d, torch.bfloat16, 4)
    clean = [t.clone() for t in lib.rms_norm(x, w, EPS, residual=res)]
    q0, s0, _ = lib.rms_norm_rows(x, w, EPS, residual=res)
    x[4, d // 3] = value
    got = lib.rms_norm(x, w, EPS, residual=res)
    keep = [i for i in range(9) if i != 4]
    for a, b in zip(got, clean):
        assert torch.equal(a[keep], b[keep])
    assert torch.isnan(got[0][4, d // 3])
    q, s, _ = lib.rms_norm_rows(x, w, EPS, residual=res)
    assert torch.equal(q[keep], q0[keep]) and torch.equal(s[keep], s0[keep]) and torch.isnan(s[4]) and not q[4].any()


def test_rows_of_zeros(lib):
    w = torch.ones(528, device="cuda")
    h, s, rstd = lib.rms_norm(torch.zeros(3, 528, device="cuda"), w, 0.25)
    assert not h.any() and (rstd == 2).all()
    q, scale, _ = lib.rms_norm_rows(torch.zeros(3, 528, device="cuda"), w, 0.25)
    assert not q.any() and not scale.any()


def test_on_another_stream_and_in_a_graph(lib):
    x, res, w, dh, dsum = _rows(37, 1032, torch.bfloat16, 8)
    h, s, rstd = lib.rms_norm(x, w, EPS, residual=res)
    dx, dw = lib.rms_norm_bwd(dh, s, w, rstd, dsum=dsum)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a = lib.rms_norm(x, w, EPS, residual=res, stream=side)
    b = lib.rms_norm_bwd(dh, a[1], w, a[2], dsum=dsum, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(a[0], h) and torch.equal(b[0], dx) and torch.equal(b[1], dw)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        g = lib.rms_norm(x, w, EPS, residual=res)
        gb = lib.rms_norm_bwd(dh, g[1], w, g[2], dsum=dsum)
    for i in range(3):
        x.copy_(torch.randn_like(x))
        graph.replay()
        want = lib.rms_norm(x, w, EPS, residual=res)
        want_b = lib.rms_norm_bwd(dh, want[1], w, want[2], dsum=dsum)
        torch.cuda.synchronize()
        for p, q in zip(g + gb, want + want_b):
            assert torch.equal(p, q), i


@pytest.mark.parametrize("N,d,lead", [(6, 520, (2, 3)), (5, 1032, (5,))])
def test_autograd(lib, N, d, lead):
    from paper_2505_24034_amd.autograd import rms_norm
    x0, r0, w0, dh, dsum = _rows(N, d, torch.float32, 12)
    for use_sum in (True, False):
        x, r, w = (t.clone().requires_grad_() for t in (x0.view(*lead, d), r0.view(*lead, d), w0))
        h, s = rms_norm(x, w, EPS, residual=r)
        assert h.shape == x.shape
        ((h * dh.view(*lead, d)).sum() + ((s * dsum.view(*lead, d)).sum() if use_sum else 0)).backward()
        want, want_dw = rms_bwd(f64(dh), f64(x0) + f64(r0), f64(w0), EPS, f64(dsum) if use_sum else None)
        scale = np.abs(want).max()
        assert torch.equal(x.grad, r.grad) and np.abs(f64(x.grad).reshape(N, d) - want).max() <= 100 * U * scale
        assert np.abs(f64(w.grad) - want_dw).max() <= 100 * U * N * np.abs(want_dw).max()
    # the sum alone; a gradient that is one number spread out; a weight that is not trained
    x, r, w = (t.clone().requires_grad_() for t in (x0, r0, w0))
    rms_norm(x, w, EPS, residual=r)[1].sum().backward()
    assert (x.grad == 1).all() and (r.grad == 1).all() and (w.grad is None or not w.grad.any())
    x = x0.clone().requires_grad_()
    rms_norm(x, w0, EPS).sum().backward()
    want, _ = rms_bwd(np.ones((N, d)), f64(x0), f64(w0), EPS)
    assert np.abs(f64(x.grad) - want).max() <= 100 * U * np.abs(want).max() + 100 * U
    with torch.no_grad():
        assert torch.equal(rms_norm(x, w0, EPS), lib.rms_norm(x0, w0, EPS)[0])


def test_a_gradient_of_a_gradient_is_refused(lib):
    from paper_2505_24034_amd.autograd import rms_norm
    x0, r0, w0, _, _ = _rows(3, 64, torch.float32, 13)
    x, r, w = (t.clone().requires_grad_() for t in (x0, r0, w0))
    h, s = rms_norm(x, w, EPS, residual=r)
    dx, = torch.autograd.grad((h * h).sum() + (s * s).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        ((dx * dx).sum() + (x * x).sum()).backward()
