"""The generator's operators as they follow one another: the residual stream of the drafted places is normalised to int8, multiplied with the head,
the drafts are verified, and the log-probabilities that come out are the trainer's mu.  Each step is held to its plain form on what the step before gave."""
import numpy as np
import pytest
import torch

from generator_util import U, quantise_rows, rms, row_logits, verify
from operator_util import f64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,K,d,V,out", [(1, 4, 1040, 3001, torch.float32), (7, 3, 528, 5003, torch.bfloat16), (24, 5, 272, 9000, torch.float32)])
def test_drafting_step(lib, B, K, d, V, out):
    g = torch.Generator().manual_seed(B)
    N = B * (K + 1)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    x, res, w = r(N, d).bfloat16().cuda(), r(N, d).bfloat16().cuda(), (1 + 0.2 * r(d)).bfloat16().cuda()
    W = (r(V, d) * 2 * d ** -0.5).bfloat16().cuda()
    Wq, Ws = lib.quantise_rows(W)
    want_q, want_s = quantise_rows(W.float().cpu().numpy())
    assert np.array_equal(Wq.cpu().numpy(), want_q) and np.array_equal(Ws.cpu().numpy(), want_s)
    q, scale, s = lib.rms_norm_rows(x, w, 1e-5, residual=res)
    h = rms(f64(s), f64(w), 1e-5)[0]
    assert (np.abs(f64(q) * f64(scale)[:, None] - h) <= f64(scale)[:, None] * (0.5 + 127 * 14 * U)).all()
    z = lib.logits_rows(q, scale, Wq, Ws, dtype=out)
    want = torch.from_numpy(row_logits(q.cpu().numpy(), scale.cpu().numpy(), want_q, want_s)).to(out)
    assert torch.equal(z.cpu(), want)
    # drafts: the head's own of a neighbouring place, some of them likely, some not
    drafts = z.view(B, K + 1, V)[:, :K].float().add(torch.randn(B, K, V, generator=g).cuda()).argmax(dim=2).to(torch.int32)
    u = (torch.rand(B, K + 1, generator=g) * (1 - 2.0 ** -24)).cuda()
    tokens, accepted, logp = lib.verify_drafts(z, drafts, u)
    ref = verify(want.float().numpy().reshape(B, K + 1, V), drafts.cpu().numpy(), u.cpu().numpy())
    assert np.array_equal(tokens.cpu().numpy(), ref[0]) and np.array_equal(accepted.cpu().numpy(), ref[1])
    assert (np.abs(f64(logp) - ref[2]) <= U * np.abs(ref[2]) + 1e-11).all()
    # under the same head, the fused log-probabilities of the tokens are the same numbers (fp32 logits)
    mask = (tokens.reshape(-1) >= 0).to(torch.uint8)
    mu, lse = lib.token_logprobs_rows(q, scale, Wq, Ws, tokens.reshape(-1), mask)
    if out == torch.float32:
        assert float((mu - logp.reshape(-1)).abs().max()) <= U * (6 * float(z.abs().max()) + 400 + 2 * float(lse.abs().max()))
    # and the trainer takes them as mu: the ratio of the policy to itself is 1
    adv = torch.ones(B, device="cuda")
    loss, coef, stats = lib.offpolicy_loss_fwd(logp.reshape(-1), logp.reshape(-1), adv, mask, B, K + 1)
    assert float(stats[0]) == float(mask.sum()) and np.allclose(f64(coef)[f64(mask) != 0], -1 / float(mask.sum()), rtol=1e-6)
