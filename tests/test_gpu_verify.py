"""Drafted tokens against the target's logits.  Tokens and counts are those of the plain form, whole numbers; the kernels decide in 64 bits, so a number
that falls within 1e-12 of a border, the only one that could differ, does not come up in these inputs.  A log-probability is a 64-bit value
rounded once: u of itself, and 1e-12 of what the exponentials leave."""
import numpy as np
import pytest
import torch

from generator_util import U, verify

pytestmark = pytest.mark.gpu


def _inputs(B, K, V, dtype, seed, model=True, greedy=0.25, size=2.0):
    g = np.random.default_rng(seed)
    z = torch.from_numpy(size * g.standard_normal((B, K + 1, V))).to(dtype)
    y = torch.from_numpy(z[:, :K].float().numpy() + 0.7 * g.standard_normal((B, K, V))).to(dtype) if model else None
    source = (y if model else z[:, :K]).float().numpy()
    drafts = (source + g.gumbel(size=(B, K, V))).argmax(axis=2).astype(np.int32) if K else np.zeros((B, 0), dtype=np.int32)
    temps = np.where(g.random(B) < greedy, 0, 0.5 + g.random(B)).astype(np.float32)
    lens = g.integers(0, K + 1, B).astype(np.int32)
    u = g.random((B, K + 1)).astype(np.float32)
    return z, y, drafts, np.minimum(u, np.float32(1 - 2.0 ** -24)), lens, temps


def _run(lib, z, y, drafts, u, lens, temps, **kw):
    c = lambda t: None if t is None else (t if torch.is_tensor(t) else torch.from_numpy(t)).cuda()  # noqa: E731
    return lib.verify_drafts(c(z), c(drafts), c(u), draft_logits=c(y), draft_lens=c(lens), temperature=c(temps), **kw)


def _check(got, z, y, drafts, u, lens, temps):
    want = verify(z.float().numpy(), drafts, u, None if y is None else y.float().numpy(), lens, temps)
    tokens, accepted, logp = (t.cpu().numpy() for t in got)
    assert np.array_equal(accepted, want[1]) and np.array_equal(tokens, want[0])
    bad = np.isnan(want[2])
    assert np.array_equal(bad, np.isnan(logp))
    assert (np.abs(logp - want[2])[~bad] <= (U * np.abs(want[2]) + 1e-11)[~bad]).all()


SIZES = [(1, 0, 1), (1, 0, 7), (1, 1, 1), (3, 2, 5), (7, 3, 5003), (2, 4, 8192), (2, 4, 8193), (4, 8, 20011), (64, 5, 1000), (1, 4, 128256), (5, 127, 33),
         (1025, 1, 17), (2, 17, 40000), (2, 2, 140001), (1, 1, 700001)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("model", [True, False])
@pytest.mark.parametrize("B,K,V", SIZES)
def test_tokens(lib, B, K, V, model, dtype):
    x = _inputs(B, K, V, dtype, B + K + V, model and K > 0)
    got = _run(lib, *x)
    _check(got, *x)
    need = lib.verify_drafts_workspace_bytes(B, K, V)
    again = _run(lib, *x, ws=torch.full((need,), 255, dtype=torch.uint8, device="cuda"))
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    z, y, drafts, u, _, _ = x                                              # all drafts, T = 1, rows as a head's logits come
    _check(_run(lib, z.reshape(-1, V), None if y is None else y.reshape(-1, V), drafts, u, None, None), z, y, drafts, u, None, None)


@pytest.mark.parametrize("model", [True, False])
def test_masked_logits(lib, model):
    """tokens that are banned for one or both, rows with one token left, with none, with NaN and infinities"""
    g = np.random.default_rng(5)
    z, y, drafts, u, lens, temps = _inputs(40, 3, 9000, torch.float32, 77, model, greedy=0.2)
    lens[:] = 3
    z[:, :, :4000] = -np.inf                                               # a whole part of the vocabulary, and then some
    z[torch.from_numpy(g.random(z.shape) < 0.5)] = -np.inf
    z[0, 0], z[1, 1], z[2, 3] = -np.inf, -np.inf, -np.inf
    z[3, 0, 17], z[4, 1, 8999], z[5, 0, 0] = np.nan, np.nan, np.inf
    z[6, 0] = -np.inf
    z[6, 0, 8500] = 3.0                                                    # one left
    z[7, 1, 8191:8193] = 50.0                                              # a tie across the border of two chunks
    drafts[6, 0], temps[7] = 8500, 0.0
    if model:
        y[8, 0], y[9, 1, 5], y[10, 0, 9] = -np.inf, np.nan, np.inf
        y[11, 0] = -np.inf
        y[11, 0, drafts[11, 0]] = 0.0
        y[12:20] = z[12:20, :3]                                            # the target's own drafts
    drafts[21, 0], drafts[22, 1], drafts[23, 2] = -1, 9000, 2 ** 31 - 1
    _check(_run(lib, z, y, drafts, u, lens, temps), z, y, drafts, u, lens, temps)


def test_drafts_of_the_target_itself_are_all_accepted(lib):
    z, _, drafts, u, _, temps = _inputs(50, 4, 700, torch.bfloat16, 8, False, greedy=0.0)
    z[0, 0, int(drafts[0, 0])] = -np.inf                                   # but for one that neither allows: p = q, nothing is left, p it is
    got = _run(lib, z, z[:, :4].contiguous(), drafts, u, None, temps)
    _check(got, z, z[:, :4].contiguous(), drafts, u, None, temps)
    assert got[1][0] == 0 and int(got[0][0, 0]) >= 0 and (got[1][1:] == 4).all()


@pytest.mark.parametrize("V", [5, 333, 9001])
@pytest.mark.parametrize("T", [-1.0, float("nan"), float("inf"), 1e-30, 1e-3, 1e30])
def test_temperatures(lib, T, V):
    z, y, drafts, u, lens, temps = _inputs(6, 3, V, torch.float32, 9)
    temps[:] = np.float32(T)
    _check(_run(lib, z, y, drafts, u, lens, temps), z, y, drafts, u, lens, temps)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [300, 9001])
def test_masks_of_the_lowest_number(lib, V, dtype):
    """the type's lowest number is a token that is never drawn, unless a row holds nothing else; logits as large as the type's come out as T = 0 does"""
    z, y, drafts, u, lens, temps = _inputs(12, 2, V, dtype, 21, greedy=0.0)
    low, high = torch.finfo(dtype).min, torch.finfo(dtype).max
    z[:, :, :V // 3] = low
    y[:, :, V // 2:] = low
    z[2], y[3] = low, low
    z[4] = -float("inf")
    z[4, :, 7:20] = low
    z[5, 0, V // 2], z[6, 1] = high, high
    lens[:] = 2
    _check(_run(lib, z, y, drafts, u, lens, temps), z, y, drafts, u, lens, temps)
    z[:, :, :V // 3] = torch.where(torch.isinf(z[:, :, :V // 3]), z[:, :, :V // 3], torch.full((), -1e4, dtype=dtype))      # far enough
    _check(_run(lib, z, y, drafts, u, lens, temps), z, y, drafts, u, lens, temps)


def test_numbers_and_lengths_at_their_ends(lib):
    z, y, drafts, u, lens, temps = _inputs(12, 3, 501, torch.float32, 10, greedy=0.2)
    lens[:4] = [-5, 99, 0, 2 ** 31 - 1]
    u[:, 3] = [0.0, 1 - 2.0 ** -24, 1.0, -3.0, np.nan, np.inf, 2.0 ** -149, 0.5, 0.25, 1.5, 0.0, 1 - 2.0 ** -24]
    u[:, 0] = [0.0, 0.0, 1.0, 2.0, -1.0, np.nan, 0.0, 1 - 2.0 ** -24, 0.5, 0.5, np.inf, 0.0]
    _check(_run(lib, z, y, drafts, u, lens, temps), z, y, drafts, u, lens, temps)


def test_first_tokens_have_the_target_s_distribution(lib):
    g = np.random.default_rng(4)
    B, V = 60000, 7
    z, y = 1.5 * g.standard_normal(V), 1.5 * g.standard_normal(V)
    drafts = (y + g.gumbel(size=(B, 1, V))).argmax(axis=2).astype(np.int32)
    spread = lambda a, n: torch.from_numpy(np.tile(a, (B, n, 1))).float()  # noqa: E731
    tokens, _, _ = _run(lib, spread(z, 2), spread(y, 1), drafts, g.random((B, 2)).astype(np.float32) * np.float32(1 - 2.0 ** -23), None, None)
    p = np.exp(z) / np.exp(z).sum()
    freq = np.bincount(tokens[:, 0].cpu().numpy(), minlength=V) / B
    assert (np.abs(freq - p) < 5 * np.sqrt(p * (1 - p) / B)).all()


def test_on_another_stream_and_in_a_graph(lib):
    z, y, drafts, u, lens, temps = (None if t is None else (t if torch.is_tensor(t) else torch.from_numpy(t)).cuda()
                                    for t in _inputs(9, 4, 9001, torch.bfloat16, 11))
    call = lambda **kw: lib.verify_drafts(z, drafts, u, draft_logits=y, draft_lens=lens, temperature=temps, **kw)  # noqa: E731
    want = call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = call(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for i in range(4):
        z.copy_(2 * torch.randn(z.shape, device="cuda"))
        u.copy_(torch.rand(u.shape, device="cuda"))
        graph.replay()
        want = call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), i
