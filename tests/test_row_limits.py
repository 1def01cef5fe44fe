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


@no_gpu_only
@pytest.mark.parametrize("cols,most", QUANTISE)
def test_rows_of_quantise_rows(cols, most):
    lib = L.load()

    def call(rows, dt):
        return lib.llamarl_quantise_rows(vp(A), rows, cols, dt, vp(A), vp(A), None)

    for dt in (L.F32, L.BF16):
        assert call(most, dt) == L.ERR_INVALID_ARG and b"overlap" in lib.llamarl_last_error()
        assert call(most + 1, dt) == L.ERR_UNSUPPORTED
