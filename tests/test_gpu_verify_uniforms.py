"""Numbers of 1 and more draw what the largest fp32 number below 1 draws: not the row's last token, which may have next to no probability."""
import numpy as np
import pytest
import torch

from test_gpu_verify import _check, _run

pytestmark = pytest.mark.gpu
BELOW_1 = np.float32(1 - 2.0 ** -24)


@pytest.mark.parametrize("model", [True, False])
@pytest.mark.parametrize("V", [6, 501, 20011])
def test_last_tokens_of_next_to_no_probability(lib, V, model):
    g = np.random.default_rng(V)
    ends = np.array([1.0, np.inf, 1 + 2.0 ** -23, 3.4e38, BELOW_1], dtype=np.float32)
    B = 8 * len(ends)
    z = g.standard_normal((B, 2, V)).astype(np.float32)
    z[:, :, V // 2:] -= 45.0                                               # less than 1e-15 together, each more than 0
    y = (z[:, :1] + g.standard_normal((B, 1, V))).astype(np.float32) if model else None
    drafts = g.integers(0, V // 2, (B, 1)).astype(np.int32)
    u = np.stack([g.random(B).astype(np.float32) * BELOW_1, np.tile(ends, 8)], axis=1)
    lens = (np.arange(B) // len(ends) % 2).astype(np.int32)                # half of them without a draft
    x = torch.from_numpy(z), None if y is None else torch.from_numpy(y), drafts
    got = _run(lib, *x, u, lens, None)
    _check(got, *x, u, lens, None)
    last = got[0].gather(1, got[1].long()[:, None]).cpu().numpy()[:, 0]
    assert (last < V // 2).all()
    capped = _run(lib, *x, np.minimum(u, BELOW_1), lens, None)
    assert all(torch.equal(a, b) for a, b in zip(got, capped))


@pytest.mark.parametrize("model", [True, False])
def test_a_draft_s_number_is_compared_as_it_is(lib, model):
    g = np.random.default_rng(1)
    values = np.array([1.0, 1.25, 3.4e38, np.inf, np.nan, BELOW_1], dtype=np.float32)
    B, V = 20 * len(values), 9
    z, y = 2 * g.standard_normal((B, 2, V)).astype(np.float32), 2 * g.standard_normal((B, 1, V)).astype(np.float32)
    drafts = z[:, :1].argmax(axis=2).astype(np.int32)
    u = np.stack([np.tile(values, 20), g.random(B).astype(np.float32) * BELOW_1], axis=1)
    x = torch.from_numpy(z), torch.from_numpy(y) if model else None, drafts, u, None, None
    got = _run(lib, *x)
    _check(got, *x)
    assert not got[1].cpu().numpy()[~np.isfinite(np.tile(values, 20))].any()
    if model:
        assert got[1].cpu().numpy()[np.tile(values, 20) == 1].any()
