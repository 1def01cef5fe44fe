"""How many rows a call may have: what a launch of its own threads holds.  Without a GPU: a size that is taken fails at its next check, here of arrays that
overlap."""
import ctypes

import pytest
import torch

from paper_2505_24034_amd import binding as L

no_gpu_only = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="fake device pointers: CPU-only test")
vp = ctypes.c_void_p
A = 1 << 32
# columns, and the most rows that quantise_rows takes of them
QUANTISE = [(16, 2 ** 26 - 4), (1024, 2 ** 26 - 4), (1040, 2 ** 24 - 1), (4096, 2 ** 24 - 1), (8192, 2 ** 24 - 1), (8208, 2 ** 22 - 1), (16400, 2 ** 22 - 1),
            (131056, 2 ** 22 - 1)]
NORM = [(8, 2 ** 26 - 4), (1024, 2 ** 26 - 4), (1032, 2 ** 24 - 1), (2048, 2 ** 24 - 1), (2056, 2 ** 23 - 1), (4096, 2 ** 23 - 1), (4104, 2 ** 22 - 1),
        (16384, 2 ** 22 - 1)]


@no_gpu_only
@pytest.mark.parametrize("cols,most", QUANTISE)
def test_rows_of_quantise_rows(cols, most):
    lib = L.load()

    def call(rows, dt):
        return lib.llamarl_quantise_rows(vp(A), rows, cols, dt, vp(A), vp(A), None)

    for dt in (L.F32, L.BF16):
        assert call(most, dt) == L.ERR_INVALID_ARG and b"overlap" in lib.llamarl_last_error()
        assert call(most + 1, dt) == L.ERR_UNSUPPORTED


@no_gpu_only
@pytest.mark.parametrize("d,most", NORM)
def test_rows_of_the_norm(d, most):
    lib = L.load()

    def forward(N, dt, out=0):
        scale = vp(A) if out else None
        return lib.llamarl_rms_norm(vp(A), vp(A), vp(A), N, d, dt, L.F32, 1e-5, out, vp(A), vp(A), scale, vp(A), None)

    def backward(N, dt):
        return lib.llamarl_rms_norm_bwd(vp(A), vp(A), vp(A), vp(A), vp(A), N, d, dt, L.F32, vp(A), None, L.F32, None, 0, None)

    for dt in (L.F32, L.BF16):
        for call in (forward, backward) + ((lambda N, dt: forward(N, dt, 1), lambda N, dt: forward(N, dt, 2)) if d % 16 == 0 else ()):
            assert call(most, dt) == L.ERR_INVALID_ARG and b"overlap" in lib.llamarl_last_error()
            assert call(most + 1, dt) == L.ERR_UNSUPPORTED


@no_gpu_only
def test_sizes_of_verify_drafts():
    lib = L.load()

    def call(B, K, V):
        return lib.llamarl_verify_drafts(vp(A), None, vp(A), None, None, vp(A), B, K, V, L.F32, vp(A), vp(A), vp(A), vp(A), 1 << 62, None)

    # B (2 K + 1) ceil(V / 8192) on either side of 2^24, and the other bounds
    for B, K, V in ((2 ** 24 // 255, 127, 8192), (2 ** 20 - 1, 7, 8192), (2 ** 24 // (3 * 256), 1, 2 ** 21 - 1), (2 ** 20 - 1, 0, 16 * 8192), (1, 127, 2 ** 21 - 1)):
        taken = B * (2 * K + 1) * -(-V // 8192) < 2 ** 24
        assert (call(B, K, V) == (L.ERR_INVALID_ARG if taken else L.ERR_UNSUPPORTED)) and (L.verify_drafts_workspace_bytes(B, K, V) > 0) == taken, (B, K, V)
    for B, K, V in ((2 ** 24 // 255 + 1, 127, 8192), (2 ** 24 // 255, 127, 8193), (2 ** 20, 0, 1), (1, 128, 1), (1, 0, 2 ** 21)):
        assert call(B, K, V) == L.ERR_UNSUPPORTED and L.verify_drafts_workspace_bytes(B, K, V) == 0


@no_gpu_only
def test_tiles_of_the_head_in_integers():
    lib = L.load()

    def call(N, V):
        return lib.llamarl_logits_rows(vp(A), vp(A), vp(A), vp(A), N, 16, V, L.F32, vp(A), None)

    for N in (2 ** 16 * 64, 2 ** 26):
        V = 2 ** 31 // (N // 64) * 64
        assert V > 2 ** 21 or call(N, V) == L.ERR_UNSUPPORTED
        assert call(N, min(V - 64, 2 ** 21 - 1)) == L.ERR_INVALID_ARG and b"overlap" in lib.llamarl_last_error()
