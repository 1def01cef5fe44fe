"""Logits that are NaN reach the log-sum-exp they belong to, also where they fill a vocabulary tile by themselves: the maximum of such a
tile passes over them, and only the sum of exponentials shows them."""
import numpy as np
import pytest
import torch

from operator_util import make_blocks

pytestmark = pytest.mark.gpu
V = 8193                                                                   # one row in the last tile, whatever the tiles' size


def _inputs(N, seed):
    g = np.random.default_rng(seed)
    targets = torch.from_numpy(g.integers(0, V - 1, N).astype(np.int32)).cuda()
    mask = torch.from_numpy((np.arange(N) % 5 != 2).astype(np.uint8)).cuda()
    return targets, mask, g


def _check(clean, bad_h, bad_w, mask, row, apart=0.0):
    """bad_h: token `row` is NaN; bad_w: the last row of W is; apart: what the other tokens may differ by"""
    on = mask != 0
    assert on[row] and torch.isfinite(clean[0]).all() and torch.isfinite(clean[1]).all()
    others = torch.arange(len(mask), device="cuda") != row
    for good, bad in zip(clean, bad_h):
        assert torch.isnan(bad[row]) and ((bad - good).abs()[others] <= apart).all()
    for bad in bad_w:
        assert torch.isnan(bad[on]).all() and (bad[~on] == 0).all()


# the kernels for few tokens (two), tiles of 64, 128 and 256 rows
@pytest.mark.parametrize("N,d,kernel", [(3, 4096, 0), (12, 144, 1), (40, 144, 1), (70, 144, 2), (130, 144, 3), (1600, 144, 4)])
def test_8_bit_head(lib, N, d, kernel):
    assert lib._load_native().block_plan(N, V, d, 0)[0] == kernel
    targets, mask, g = _inputs(N, N)
    x = (*make_blocks(g.standard_normal((N, d)), 1, "cuda"), *make_blocks(g.standard_normal((V, d)) * d ** -0.5, 128, "cuda"))
    row = N - 1 if (N - 1) % 5 != 2 else N - 2

    def call():
        return lib.token_logprobs_blocks(*x, targets, mask)

    def with_nan(q, at):
        code = q.view(torch.uint8)[at].clone()
        q.view(torch.uint8)[at] = 0x7F
        out = call()
        q.view(torch.uint8)[at] = code
        return out

    _check(call(), with_nan(x[0], row), with_nan(x[2], V - 1), mask, row)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [3, 130, 1100])
def test_head_and_its_shards(lib, N, dtype):
    d = 64
    targets, mask, g = _inputs(N, N)
    H = torch.from_numpy(g.standard_normal((N, d))).to(dtype).cuda()
    W = torch.from_numpy(g.standard_normal((V, d)) * d ** -0.5).to(dtype).cuda()
    row = N - 1 if (N - 1) % 5 != 2 else N - 2

    def whole():
        return lib.token_logprobs(H, W, targets, mask)

    def shards():
        parts = [lib.token_logprobs_partial(H, W[a:b].contiguous(), targets, a, V, mask) for a, b in ((0, 4096), (4096, V - 1), (V - 1, V))]
        return lib.merge_partials(*(torch.stack(p) for p in zip(*parts)))

    # An fp32 tile with a NaN is contracted again in another order: two fp32 sums, each within 4 (sqrt(d) + 4) u of its products' root sum of
    # squares, which |h|_max |w| bounds, and 16 u (|lse| + |logp| + 8) for exponentials, logarithm and merge.  bf16: the same bits.
    apart = 0.0
    if dtype == torch.float32:
        rss = float(H.abs().max() * W.norm(dim=1).max())
        logp, lse = whole()
        apart = 2 * 2.0 ** -24 * (4 * (d ** 0.5 + 4) * rss + 16 * float(lse.max() - logp.min() + 8))
    for call in (whole, shards):
        clean = call()
        outs = []
        for x, at in ((H, row), (W, V - 1)):
            kept = x[at].clone()
            x[at] = float("nan")
            outs.append(call())
            x[at] = kept
        _check(clean, *outs, mask, row, apart)
