"""What the norm, the head in 8-bit integers and the verification of drafts refuse, without a GPU: every check comes before anything is launched."""
import ctypes

import pytest
import torch

from paper_2505_24034_amd import binding as L

no_gpu_only = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="fake device pointers: CPU-only test")
NAN, INF = float("nan"), float("inf")
vp = ctypes.c_void_p
A = 1 << 32


@pytest.fixture(scope="module")
def clib():
    return L.load()


@no_gpu_only
def test_quantise_rows(clib):
    def call(x=A, rows=10, cols=64, dt=L.BF16, q=2 * A, scale=3 * A):
        return clib.llamarl_quantise_rows(vp(x), rows, cols, dt, vp(q), vp(scale), None)

    for bad in (dict(x=None), dict(q=None), dict(scale=None), dict(rows=0), dict(cols=0), dict(rows=-1), dict(dt=2), dict(x=A + 8), dict(q=2 * A + 4),
                dict(scale=3 * A + 2), dict(q=A + 16), dict(scale=A + 1276), dict(scale=2 * A + 636)):
        assert call(**bad) == L.ERR_INVALID_ARG, bad
    for bad in (dict(cols=24), dict(cols=1 << 17), dict(rows=1 << 31), dict(rows=1 << 23, cols=16384), dict(rows=1 << 24, cols=4096)):
        assert call(**bad) == L.ERR_UNSUPPORTED, bad
    assert b"" != clib.llamarl_last_error()


@no_gpu_only
def test_logits_rows(clib):
    def call(H=A, hs=2 * A, W=3 * A, ws=4 * A, N=10, d=64, V=100, dt=L.F32, z=5 * A):
        return clib.llamarl_logits_rows(vp(H), vp(hs), vp(W), vp(ws), N, d, V, dt, vp(z), None)

    for bad in (dict(H=None), dict(hs=None), dict(W=None), dict(ws=None), dict(z=None), dict(N=0), dict(d=0), dict(V=0), dict(V=-3), dict(dt=2),
                dict(H=A + 8), dict(W=3 * A + 1), dict(hs=2 * A + 2), dict(ws=4 * A + 1), dict(z=5 * A + 4), dict(z=A + 624), dict(z=2 * A + 32),
                dict(z=3 * A - 3984), dict(z=4 * A + 384)):
        assert call(**bad) == L.ERR_INVALID_ARG, bad
    for bad in (dict(d=24), dict(d=1 << 17), dict(N=1 << 25), dict(V=1 << 21), dict(N=1 << 26, d=16, V=(1 << 21) - 1)):
        assert call(**bad) == L.ERR_UNSUPPORTED, bad


@no_gpu_only
def test_token_logprobs_rows(clib):
    need = L.logprobs_rows_workspace_bytes(10, 100)
    assert need > 0

    def call(H=A, hs=2 * A, W=3 * A, ws=4 * A, t=5 * A, mask=6 * A, N=10, d=64, V=100, logp=7 * A, lse=8 * A, scratch=9 * A, nbytes=need):
        return clib.llamarl_token_logprobs_rows(vp(H), vp(hs), vp(W), vp(ws), vp(t), vp(mask), N, d, V, vp(logp), vp(lse), vp(scratch), nbytes, None)

    for bad in (dict(t=None), dict(logp=None), dict(lse=None), dict(H=None), dict(ws=None), dict(t=5 * A + 1), dict(logp=7 * A + 2), dict(lse=8 * A + 3),
                dict(scratch=9 * A + 8), dict(lse=7 * A + 36), dict(logp=5 * A), dict(logp=6 * A + 8), dict(scratch=A), dict(scratch=7 * A - 256),
                dict(lse=2 * A), dict(logp=4 * A + 396)):
        assert call(**bad) == L.ERR_INVALID_ARG, bad
    assert call(scratch=None) == L.ERR_WORKSPACE and call(nbytes=need - 1) == L.ERR_WORKSPACE
    assert call(d=8) == L.ERR_UNSUPPORTED and call(V=1 << 21) == L.ERR_UNSUPPORTED
    for N, V in ((0, 5), (5, 0), (-1, 5), (1 << 27, 5), (5, 1 << 21)):
        assert L.logprobs_rows_workspace_bytes(N, V) == 0


def test_workspace_of_the_largest_call_serves_smaller_ones():
    for V in (1, 64, 1000, 8193, 33001, 128256):
        last = 0
        for N in range(1, 1200, 7):
            b = L.logprobs_rows_workspace_bytes(N, V)
            assert b >= last and b >= L.logprobs_rows_workspace_bytes(N, max(1, V - 77))
            last = b
    for d in (8, 2048, 4096, 16384):
        sizes = [L.rms_norm_bwd_workspace_bytes(N, d) for N in (1, 2, 5, 100, 512, 513, 1024, 5000, 100000)]
        assert sizes == sorted(sizes) and sizes[5] > 0
    last = 0
    for B, K, V in ((1, 0, 1), (1, 1, 1), (2, 1, 8192), (2, 1, 8193), (2, 9, 8193), (300, 9, 100000)):
        b = L.verify_drafts_workspace_bytes(B, K, V)
        assert b >= last > -1
        last = b


@no_gpu_only
def test_rms_norm(clib):
    def call(x=A, res=2 * A, w=3 * A, N=10, d=64, dt=L.BF16, w_dt=L.BF16, eps=1e-6, out=0, s=4 * A, h=5 * A, scale=None, rstd=7 * A):
        return clib.llamarl_rms_norm(vp(x), vp(res), vp(w), N, d, dt, w_dt, eps, out, vp(s), vp(h), vp(scale), vp(rstd), None)

    for bad in (dict(x=None), dict(w=None), dict(h=None), dict(res=None), dict(s=None), dict(N=0), dict(d=0), dict(dt=2), dict(w_dt=5), dict(eps=0.0),
                dict(eps=-1.0), dict(eps=NAN), dict(eps=INF), dict(out=3), dict(out=-1), dict(out=1), dict(out=2), dict(scale=6 * A), dict(x=A + 8),
                dict(res=2 * A + 2), dict(w=3 * A + 4), dict(s=4 * A + 8), dict(h=5 * A + 8), dict(rstd=7 * A + 1), dict(out=2, scale=6 * A + 2),
                dict(h=A + 1264), dict(s=A), dict(h=2 * A), dict(h=4 * A + 16), dict(rstd=5 * A), dict(h=3 * A + 112), dict(out=1, scale=4 * A),
                dict(out=2, scale=7 * A + 36)):
        assert call(**bad) == L.ERR_INVALID_ARG, bad
    for bad in (dict(d=12), dict(dt=L.F32, d=6), dict(d=16392), dict(out=1, scale=6 * A, d=24), dict(out=2, scale=6 * A, d=8), dict(N=1 << 31),
                dict(N=1 << 24, d=4096), dict(N=1 << 22, d=16384)):
        assert call(**bad) == L.ERR_UNSUPPORTED, bad


@no_gpu_only
def test_rms_norm_bwd(clib):
    need = L.rms_norm_bwd_workspace_bytes(600, 64)
    assert need > 0 and L.rms_norm_bwd_workspace_bytes(512, 64) == 0      # few rows need none

    def call(dh=A, s=2 * A, w=3 * A, rstd=4 * A, dsum=5 * A, N=600, d=64, dt=L.BF16, w_dt=L.BF16, dx=6 * A, dw=7 * A, dw_dt=L.F32, ws=8 * A, nbytes=need):
        return clib.llamarl_rms_norm_bwd(vp(dh), vp(s), vp(w), vp(rstd), vp(dsum), N, d, dt, w_dt, vp(dx), vp(dw), dw_dt, vp(ws), nbytes, None)

    for bad in (dict(dh=None), dict(s=None), dict(w=None), dict(rstd=None), dict(dx=None), dict(N=-1), dict(d=0), dict(dt=9), dict(w_dt=2), dict(dw_dt=2),
                dict(dh=A + 2), dict(s=2 * A + 8), dict(dsum=5 * A + 8), dict(dx=6 * A + 8), dict(rstd=4 * A + 2), dict(dw=7 * A + 2), dict(ws=8 * A + 8),
                dict(dx=A), dict(dx=5 * A + 1264), dict(dw=3 * A), dict(dw=6 * A + 4), dict(ws=6 * A - 16), dict(dx=4 * A + 32), dict(dw=8 * A + 4)):
        assert call(**bad) == L.ERR_INVALID_ARG, bad
    assert call(ws=None) == L.ERR_WORKSPACE and call(nbytes=need - 1) == L.ERR_WORKSPACE
    assert call(d=12) == L.ERR_UNSUPPORTED and call(d=16400) == L.ERR_UNSUPPORTED
    assert L.rms_norm_bwd_workspace_bytes(0, 64) == 0 and L.rms_norm_bwd_workspace_bytes(5, 0) == 0 and L.rms_norm_bwd_workspace_bytes(5, 16392) == 0


@no_gpu_only
def test_verify_drafts(clib):
    need = L.verify_drafts_workspace_bytes(4, 3, 100)

    def call(z=A, y=2 * A, x=3 * A, lens=4 * A, t=5 * A, u=6 * A, B=4, K=3, V=100, dt=L.F32, tok=7 * A, acc=8 * A, lp=9 * A, ws=10 * A, nbytes=need):
        return clib.llamarl_verify_drafts(vp(z), vp(y), vp(x), vp(lens), vp(t), vp(u), B, K, V, dt, vp(tok), vp(acc), vp(lp), vp(ws), nbytes, None)

    for bad in (dict(z=None), dict(x=None), dict(u=None), dict(tok=None), dict(acc=None), dict(lp=None), dict(B=0), dict(K=-1), dict(V=0), dict(dt=3),
                dict(z=A + 2), dict(y=2 * A + 1), dict(dt=L.BF16, z=A + 1), dict(x=3 * A + 1), dict(lens=4 * A + 2), dict(t=5 * A + 1), dict(u=6 * A + 3),
                dict(tok=7 * A + 2), dict(acc=8 * A + 1), dict(lp=9 * A + 2), dict(ws=10 * A + 8), dict(tok=A + 6396), dict(lp=3 * A), dict(acc=7 * A + 60),
                dict(tok=3 * A + 44), dict(ws=6 * A - 16), dict(acc=4 * A), dict(lp=5 * A + 12), dict(ws=2 * A)):
        assert call(**bad) == L.ERR_INVALID_ARG, bad
    assert call(ws=None) == L.ERR_WORKSPACE and call(nbytes=need - 1) == L.ERR_WORKSPACE
    for bad in (dict(K=128), dict(V=1 << 21), dict(B=1 << 20), dict(B=1 << 19, K=100, V=100000)):
        assert call(**bad) == L.ERR_UNSUPPORTED, bad
    assert L.verify_drafts_workspace_bytes(0, 1, 1) == 0 and L.verify_drafts_workspace_bytes(1, -1, 1) == 0 and L.verify_drafts_workspace_bytes(1, 128, 9) == 0


def test_binding_refuses_host_tensors():
    x, w = torch.zeros(4, 64), torch.ones(64)
    i8, s = torch.zeros(4, 64, dtype=torch.int8), torch.ones(4)
    for call in (lambda: L.quantise_rows(x), lambda: L.logits_rows(i8, s, i8, s), lambda: L.token_logprobs_rows(i8, s, i8, s, torch.zeros(4, dtype=torch.int32)),
                 lambda: L.rms_norm(x, w), lambda: L.rms_norm_rows(x, w), lambda: L.rms_norm_blocks(x, w), lambda: L.rms_norm_bwd(x, x, w, s),
                 lambda: L.verify_drafts(torch.zeros(2, 2, 8), torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 2)),
                 lambda: L.quantise_rows(x.half()), lambda: L.rms_norm(x.double(), w)):
        with pytest.raises(L.LlamarlError) as e:
            call()
        assert e.value.status == L.ERR_INVALID_ARG
    with pytest.raises(TypeError):
        L.rms_norm(None, w)


@pytest.mark.gpu
def test_binding_refuses_shapes_types_and_strides(lib):
    c = dict(device="cuda")
    x, w = torch.zeros(4, 64, **c), torch.ones(64, **c)
    q, s = torch.zeros(4, 64, dtype=torch.int8, **c), torch.ones(4, **c)
    t = torch.zeros(4, dtype=torch.int32, **c)
    z, d, u = torch.zeros(2, 3, 10, **c), torch.zeros(2, 2, dtype=torch.int32, **c), torch.zeros(2, 3, **c)
    bad = [lambda: lib.quantise_rows(x[:, ::2]), lambda: lib.quantise_rows(x.view(-1)), lambda: lib.logits_rows(q, s[:3], q, s),
           lambda: lib.logits_rows(q, s, q[:, :32].contiguous(), s), lambda: lib.logits_rows(q.to(torch.uint8), s, q, s), lambda: lib.logits_rows(q, s, q, s.double()),
           lambda: lib.logits_rows(q, s, q, s, out=torch.zeros(4, 5, **c)), lambda: lib.logits_rows(q, s, q, s, out=torch.zeros(4, 4, dtype=torch.half, **c)),
           lambda: lib.token_logprobs_rows(q, s, q, s, t[:3]), lambda: lib.token_logprobs_rows(q, s, q, s, t.long()),
           lambda: lib.token_logprobs_rows(q, s, q, s, t, torch.zeros(3, dtype=torch.uint8, **c)),
           lambda: lib.rms_norm(x, w[:32]), lambda: lib.rms_norm(x.t(), torch.ones(4, **c)), lambda: lib.rms_norm(x, w, residual=x[:2]),
           lambda: lib.rms_norm(x, w, residual=x.bfloat16()), lambda: lib.rms_norm(x, w, eps=0.0), lambda: lib.rms_norm(x, w.cpu()),
           lambda: lib.rms_norm_bwd(x, x, w, s[:2]), lambda: lib.rms_norm_bwd(x.bfloat16(), x, w, s), lambda: lib.rms_norm_bwd(x, x, w, s, dsum=x[:, :8]),
           lambda: lib.verify_drafts(z, d[:1], u), lambda: lib.verify_drafts(z[:, :2], d, u), lambda: lib.verify_drafts(z, d, u[:, :2]),
           lambda: lib.verify_drafts(z, d.long(), u), lambda: lib.verify_drafts(z, d, u, draft_logits=z), lambda: lib.verify_drafts(z, d, u, draft_lens=d),
           lambda: lib.verify_drafts(z, d, u, draft_logits=torch.zeros(2, 2, 9, **c)), lambda: lib.verify_drafts(z, d, u, temperature=s),
           lambda: lib.verify_drafts(z.half(), d, u), lambda: lib.verify_drafts(z, d, u, ws=torch.zeros(4096, dtype=torch.uint8)),
           lambda: lib.verify_drafts(z, d, u, ws=torch.zeros(4096, dtype=torch.uint8, pin_memory=True))]
    for call in bad:
        with pytest.raises(lib.LlamarlError) as e:
            call()
        assert e.value.status == lib.ERR_INVALID_ARG
    with pytest.raises(lib.LlamarlError) as e:
        lib.verify_drafts(z, d, u, ws=torch.zeros(16, dtype=torch.uint8, **c))
    assert e.value.status == lib.ERR_WORKSPACE
