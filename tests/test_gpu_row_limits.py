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
