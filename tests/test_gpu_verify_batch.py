"""Drafted tokens of a batch that gives a workgroup several chunks of 8192 logits, and several units of 2048 of the row that a sequence's last token is drawn
from.  Held to the plain form as test_gpu_verify.py's."""
import numpy as np
import pytest
import torch

from test_gpu_verify import _check, _inputs, _run

pytestmark = pytest.mark.gpu
CHUNK = 8192
# What each of them reaches: see test_verify_rules.py.
MASKED = [(64, 5, 45001, True), (128, 5, 45001, False), (256, 3, 40000, True)]
BATCHES = [(300, 3, 17000, True), (600, 2, 5000, True), (700, 2, 8000, False), (600, 1, 9001, True), (1500, 1, 3000, True), (130, 0, 150001, False)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,K,V,model", BATCHES)
def test_batches(lib, B, K, V, model, dtype):
    """ragged lengths, some at T = 0; every fourth sequence's drafts are the target's own, and where its first is outside the vocabulary nothing is left of
    p - q: the token comes out of p"""
    z, y, drafts, u, lens, temps = _inputs(B, K, V, dtype, B + V, model, size=4.0)
    if model:
        y[::4] = z[::4, :K]
        drafts[::8, 0] = -1
        lens[::8], temps[::8] = K, 0.9
    got = _run(lib, z, y, drafts, u, lens, temps)
    _check(got, z, y, drafts, u, lens, temps)
    scratch = torch.full((lib.verify_drafts_workspace_bytes(B, K, V),), 255, dtype=torch.uint8, device="cuda")
    again = _run(lib, z, y, drafts, u, lens, temps, ws=scratch)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,K,V,model", MASKED)
def test_chunks_without_a_sum(lib, B, K, V, model, dtype):
    """neighbouring chunks of which nothing is left, between ones with logits; a NaN or an infinity in one chunk only"""
    z, y, drafts, u, lens, temps = _inputs(B, K, V, dtype, B + V, model, greedy=0.2, size=5.0)
    g = np.random.default_rng(B)
    chunks = -(-V // CHUNK)
    where = np.arange(V) // CHUNK
    banned = g.random((B, K + 1, chunks)) < 0.6
    banned[np.arange(B)[:, None], np.arange(K + 1)[None, :], g.integers(0, chunks, (B, K + 1))] = False
    z[torch.from_numpy(banned[:, :, where])] = -np.inf
    if model:
        y[torch.from_numpy(banned[:, :K][:, :, where]) & (torch.arange(B) % 3 > 0)[:, None, None]] = -np.inf      # the same mask for most
    # a draft where its own row has something left
    allowed = ~banned[:, :K]
    at = np.where(allowed, g.random(allowed.shape), -1.0).argmax(axis=2)
    moved = np.minimum(at * CHUNK + g.integers(0, CHUNK, (B, K)), V - 1).astype(np.int32)
    gone = banned[np.arange(B)[:, None], np.arange(K)[None, :], where[drafts]]
    drafts = np.where(gone & (np.arange(B)[:, None] % 2 == 0), moved, drafts).astype(np.int32)
    u[::3, :K] *= np.float32(0.01)                                         # more of them accepted
    lens[:8], temps[1:6] = K, [1.0, 0.7, 0.0, 0.8, 1.3]
    z[1, 0, CHUNK + 3] = np.nan
    z[2, 1, V - 1] = np.nan
    z[3, 0, 5] = np.nan
    z[4, 0, CHUNK // 2] = np.inf
    z[5, 0] = -np.inf
    z[6, K, 2 * CHUNK:3 * CHUNK] = -np.inf
    if model:
        y[7, 0, 3 * CHUNK - 1] = np.nan
    _check(_run(lib, z, y, drafts, u, lens, temps), z, y, drafts, u, lens, temps)
