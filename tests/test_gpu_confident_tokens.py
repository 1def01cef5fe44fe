"""Log-probabilities under the 8-bit head of tokens that have most of the probability, as a trained policy's have.

Such a row's log-sum-exp is nearly its target's logit, and whatever differs between the two is left in logp.  With p the target's
probability, logp = -log(1 + R / e): the target's term e is an fp32 sum, off by 4 (sqrt(d) + 4) u of its products' root sum of squares
(rss) at most, the others' terms R come from the 8-bit pipe, and both move logp by their error times 1 - p.  Exponentials, sums and
the merge leave 16 u (|lse| + |logp| + 8).  lse = z - logp adds the target's own error once more.

The pipe cuts products, towards zero, to multiples of 2^-13 of the largest of eight: seven errors of the products' own, here random, signs and a variance
of 2^-26 max^2 / 3 at most, in all (7 / 3) 2^-26 rss^2.  2^-10 rss is five times the root of that."""
import numpy as np
import pytest
import torch

from operator_util import dequantise, f64, log_softmax_at, make_blocks

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


# the kernels for few tokens (two), tiles of 64, 128 and 256 rows
@pytest.mark.parametrize("N,d,V,kernel", [(3, 2064, 1000, 0), (50, 528, 3001, 1), (100, 528, 5003, 2), (130, 1040, 16500, 3), (300, 528, 33000, 4),
                                          (300, 2064, 24601, 4)])
def test_confident_tokens(lib, N, d, V, kernel):
    assert lib._load_native().block_plan(N, V, d, 0)[0] == kernel
    g = np.random.default_rng(N + d)
    W = g.standard_normal((V, d)) * d ** -0.5
    y = g.integers(0, V, N)
    # z of the target from 6 (one of many) to 60 (all of the probability)
    H = np.exp(g.uniform(np.log(6), np.log(60), N))[:, None] * W[y] + 0.2 * g.standard_normal((N, d))
    x = (*make_blocks(H, 1, "cuda"), *make_blocks(W, 128, "cuda"))
    logp, lse = (f64(t) for t in lib.token_logprobs_blocks(*x, torch.from_numpy(y.astype(np.int32)).cuda()))
    Hd, Wd = (torch.from_numpy(dequantise(q, s, b)).cuda() for q, s, b in ((x[0], x[1], 1), (x[2], x[3], 128)))
    z, rss = (Hd @ Wd.T).cpu().numpy(), torch.sqrt((Hd * Hd) @ (Wd * Wd).T).cpu().numpy()
    want_logp, want_lse = log_softmax_at(z, y)
    p, at = np.exp(want_logp), np.arange(N)
    assert (p > 1 - 1e-6).sum() >= N // 5 or N < 10
    target = 4 * (d ** 0.5 + 4) * U * rss[at, y]
    others = (4 * (d ** 0.5 + 4) * U if kernel <= 1 else 2.0 ** -10) * rss.max(axis=1)
    last = 16 * U * (np.abs(want_lse) + np.abs(want_logp) + 8)
    assert (np.abs(logp - want_logp) <= (1 - p) * (target + others) + last).all()
    assert (np.abs(lse - want_lse) <= target + (1 - p) * (target + others) + last).all()
    if kernel > 1:                                                         # where the target's term is formed again it never exceeds the sum
        assert (logp <= 0).all()
