"""Up to 64 tokens under the 8-bit head: sums in fp32 whatever the number of rows of W, in bf16 logits and log-probabilities too.

u = 2^-24.  A logit is off by 4 (sqrt(d) + 4) u of its products' root sum of squares (rss) at most; a bf16 one is the fp32 one
rounded.  A log-sum-exp moves by the largest of its logits' errors, and exponentials, sums and merge leave 16 u (|lse| + |logp| + 8)."""
import numpy as np
import pytest
import torch

from operator_util import dequantise, f64, log_softmax_at, make_blocks

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


# the kernels for few tokens, tiles of 64 and of 128 rows
@pytest.mark.parametrize("N,d,V,kernel", [(2, 2064, 3001, 0), (40, 528, 5003, 1), (1, 1040, 60001, 2), (3, 144, 40001, 2), (16, 528, 33003, 2),
                                          (40, 144, 66000, 2), (64, 272, 32641, 2), (33, 144, 100001, 3), (64, 528, 98500, 3)])
def test_sums_in_fp32(lib, N, d, V, kernel):
    assert lib._load_native().block_plan(N, V, d, 0)[0] == kernel
    g = np.random.default_rng(N + V)
    W = g.standard_normal((V, d)) * d ** -0.5
    y = g.integers(0, V, N)
    H = g.standard_normal((N, d))
    H[::2] = np.exp(g.uniform(np.log(10), np.log(60), len(H[::2])))[:, None] * W[y[::2]] + 0.2 * H[::2]      # rows with one likely token
    x = (*make_blocks(H, 1, "cuda"), *make_blocks(W, 128, "cuda"))
    z = lib.logits_blocks(*x)
    assert torch.equal(lib.logits_blocks(*x, dtype=torch.bfloat16), z.to(torch.bfloat16))
    Hd, Wd = (torch.from_numpy(dequantise(q, s, b)).cuda() for q, s, b in ((x[0], x[1], 1), (x[2], x[3], 128)))
    want, rss = Hd @ Wd.T, torch.sqrt((Hd * Hd) @ (Wd * Wd).T)
    sums = 4 * (d ** 0.5 + 4) * U
    assert ((z.double() - want).abs() <= sums * rss + U * want.abs()).all()
    targets = np.where(np.arange(N) % 4 == 2, g.integers(0, V, N), y)      # some of the likely tokens are not the targets
    logp, lse = (f64(t) for t in lib.token_logprobs_blocks(*x, torch.from_numpy(targets.astype(np.int32)).cuda()))
    want_logp, want_lse = log_softmax_at(want.cpu().numpy(), targets)
    off = sums * rss.amax(dim=1).cpu().numpy()
    last = 16 * U * (np.abs(want_lse) + np.abs(want_logp) + 8)
    assert (np.abs(lse - want_lse) <= off + last).all()
    assert (np.abs(logp - want_logp) <= 2 * off + last).all()


@pytest.mark.parametrize("N,V,d", [(1, 32641, 1040), (2, 40960, 1024), (1, 40945, 2048), (2, 34567, 4096)])
def test_one_or_two_tokens_straight_from_memory(lib, N, V, d):
    """the logits' kernel without LDS beside the log-probabilities' tiles"""
    assert lib._load_native().block_plan(N, V, d, 0)[0] == 2
    g = torch.Generator(device="cuda").manual_seed(V)
    H, W = torch.randn(N, d, generator=g, device="cuda"), torch.randn(V, d, generator=g, device="cuda") * d ** -0.5
    x = (*lib.quantise_blocks(H, 1), *lib.quantise_blocks(W, 128))
    out = torch.full((N + 2, V), 7.0, device="cuda").view(-1)
    off = -V % 4                                                           # 16-byte aligned rows behind the first
    z = lib.logits_blocks(*x, out=out[V + off:V + off + N * V].view(N, V))
    assert (out[:V + off] == 7).all() and (out[V + off + N * V:] == 7).all()
    Hd, Wd = (torch.from_numpy(dequantise(q, s, b)).cuda() for q, s, b in ((x[0], x[1], 1), (x[2], x[3], 128)))
    want, rss = Hd @ Wd.T, torch.sqrt((Hd * Hd) @ (Wd * Wd).T)
    assert ((z.double() - want).abs() <= 4 * (d ** 0.5 + 4) * U * rss + U * want.abs()).all()
    assert torch.equal(lib.logits_blocks(*x, dtype=torch.bfloat16), z.to(torch.bfloat16))
    t = torch.randint(0, V, (N,), generator=g, device="cuda").int()
    lse = lib.token_logprobs_blocks(*x, t)[1]
    ref = torch.logsumexp(want, 1)
    assert ((lse - ref).abs() <= 4 * (d ** 0.5 + 4) * U * rss.amax(dim=1) + 16 * U * (2 * ref.abs() + 20)).all()
