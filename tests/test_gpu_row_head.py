"""The head in 8-bit integers.  Its logits are an exact sum and three (bf16: four) roundings, which numpy does alike: they are compared bit for bit.

lse, with u = 2^-24: a term exp(z - m) is off by u of its exponent's parts (m log2 e and z log2 e - that, each below 1.45 max |z|, twice through the
merges) and a few u of the exponential; sums are chains of fewer than 64 additions, four times over."""
import numpy as np
import pytest
import torch

from generator_util import U, quantise_rows, row_logits
from operator_util import f64, log_softmax_at

pytestmark = pytest.mark.gpu


def _rng(seed):
    return np.random.default_rng(seed)


def _same(t, want):
    return np.array_equal(t.cpu().numpy(), want, equal_nan=want.dtype != np.int8)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,C", [(1, 16), (5, 512), (4, 528), (3, 1040), (9, 2048), (2, 2064), (7, 4096), (3, 8192), (2, 8208), (1, 16384), (2, 16400),
                                 (1, 131056), (1031, 48)])
def test_quantised_exactly(lib, R, C, dtype):
    g = _rng(R + C)
    x = torch.from_numpy(g.standard_normal((R, C)) * np.exp(2 * g.standard_normal((R, 1)))).to(dtype).cuda()
    q, scale = lib.quantise_rows(x)
    want, want_scale = quantise_rows(x.float().cpu().numpy())
    assert q.dtype == torch.int8 and _same(q, want) and _same(scale, want_scale)
    assert (q.abs().amax(dim=1) == 127).all()


@pytest.mark.parametrize("C", [48, 4096, 20000])
def test_quantised_borders(lib, C):
    x = np.zeros((14, C), dtype=np.float32)
    x[0] = np.arange(C) % 255 - 127.0
    x[1] = (np.arange(C) % 254 - 127.0) + 0.5                              # halves, and 126.5 the largest but for
    x[1, 0] = 127.0
    x[2, :] = 3.4028235e38
    x[2, 1] = -1e38
    x[3, 5] = 2.0 ** -100
    x[4, 5] = np.nextafter(np.float32(2.0 ** -100), np.float32(0))
    x[5, 7] = np.inf
    x[6, 9] = np.nan
    x[7, C - 1] = -np.inf
    x[8, :] = 1e-45
    x[9] = np.float32(2.0 ** -100) * (np.arange(C) % 7)
    x[10, C - 1] = -5.0
    x[11] = np.float32(1 / 3)
    x[12] = 254 * (np.arange(C) % 255 / np.float32(254))
    x[13, :] = np.ldexp(np.float32(1), -(np.arange(C) % 20))
    q, scale = lib.quantise_rows(torch.from_numpy(x).cuda())
    want, want_scale = quantise_rows(x)
    assert _same(q, want) and _same(scale, want_scale)


def _head(N, d, V, seed):
    g = _rng(seed)
    H, W = g.integers(-127, 128, (N, d), dtype=np.int8), g.integers(-127, 128, (V, d), dtype=np.int8)
    hs = np.exp(0.5 * g.standard_normal(N)).astype(np.float32) / 127
    ws = (np.exp(0.5 * g.standard_normal(V)) * d ** -0.5 / 40).astype(np.float32)
    return H, hs, W, ws


def _cuda(*xs):
    return [torch.from_numpy(x).cuda() for x in xs]


# (N, V, d): every kernel is among them, see test_row_rules.py
PRODUCTS = [(1, 5, 16), (1, 1000, 4096), (2, 300, 8208), (7, 1031, 528), (16, 4000, 1040), (16, 130, 48), (17, 70, 16), (33, 1000, 528), (48, 5003, 2064),
            (64, 64, 4096), (129, 600, 272), (300, 2000, 1040), (40, 30000, 272), (64, 17000, 1168), (128, 9000, 144), (65, 33001, 144), (128, 40000, 528),
            (100, 33000, 272), (513, 8200, 208), (300, 33001, 528), (1300, 9000, 1168), (257, 50000, 144), (3000, 5003, 272), (200, 66001, 528), (300, 50000, 784),
            (9, 33001, 1040), (3, 33001, 2064)]


@pytest.mark.parametrize("N,V,d", PRODUCTS)
def test_logits_bit_for_bit(lib, N, V, d):
    H, hs, W, ws = _head(N, d, V, N + V)
    want = row_logits(H, hs, W, ws)
    args = _cuda(H, hs, W, ws)
    z = lib.logits_rows(*args)
    assert z.dtype == torch.float32 and _same(z, want)
    out = torch.full((N + 1, V), 7.0, dtype=torch.bfloat16, device="cuda")
    assert lib.logits_rows(*args, out=out[:N]).data_ptr() == out.data_ptr()
    assert torch.equal(out[:N].cpu(), torch.from_numpy(want).to(torch.bfloat16)) and (out[N] == 7).all()
    out = torch.full((N + 1, V), 7.0, device="cuda")
    lib.logits_rows(*args, out=out[:N])
    assert _same(out[:N], want) and (out[N] == 7).all()


def test_largest_sums(lib):
    """d at its limit, every product 127 * 127 (and -128 * -128: int8 holds it, though the quantiser does not make it)"""
    d = 131056
    H, W = np.full((18, d), 127, dtype=np.int8), np.full((20, d), -127, dtype=np.int8)
    W[3], H[2] = -128, -128
    one = np.ones(20, dtype=np.float32)
    for N in (3, 18):
        assert _same(lib.logits_rows(*_cuda(H[:N], one[:N], W, one)), row_logits(H[:N], one[:N], W, one))


@pytest.mark.parametrize("N,V,d", PRODUCTS + [(1, 128256, 64), (40, 16032, 1040), (16, 20011, 2064)])
def test_logprobs(lib, N, V, d):
    H, hs, W, ws = _head(N, d, V, N * V)
    g = _rng(N)
    targets = g.integers(0, V, N).astype(np.int32)
    mask = (g.random(N) < 0.7).astype(np.uint8)
    if N > 4:
        targets[1], targets[2], targets[3] = -1, V, V - 1
        mask[:4] = 1
    args = _cuda(H, hs, W, ws, targets)
    z = row_logits(H, hs, W, ws).astype(np.float64)
    want, want_lse = log_softmax_at(z, np.clip(targets, 0, V - 1))
    for m in (mask, None):
        live = (targets >= 0) & (targets < V) & (mask != 0 if m is not None else True)
        logp, lse = lib.token_logprobs_rows(*args, None if m is None else torch.from_numpy(m).cuda())
        tol = U * (6 * np.abs(z).max(axis=1) + 300 + np.abs(want_lse))
        assert (np.abs(f64(lse) - want_lse)[live] <= tol[live]).all()
        assert (np.abs(f64(logp) - want)[live] <= (tol + U * np.abs(want))[live]).all()
        assert not f64(lse)[~live].any() and not f64(logp)[~live].any()
    ws_bytes = lib.logprobs_rows_workspace_bytes(N, V)
    scratch = torch.full((ws_bytes,), 255, dtype=torch.uint8, device="cuda")          # NaN bits everywhere
    again = lib.token_logprobs_rows(*args, None, ws=scratch)
    assert torch.equal(again[0], logp) and torch.equal(again[1], lse)


def test_all_masked(lib):
    H, hs, W, ws = _head(40, 64, 300, 1)
    logp, lse = lib.token_logprobs_rows(*_cuda(H, hs, W, ws, np.zeros(40, dtype=np.int32), np.zeros(40, dtype=np.uint8)))
    assert not logp.any() and not lse.any()


@pytest.mark.parametrize("N,V", [(5, 1000), (40, 1000), (200, 33001)])
def test_scales_that_are_not_finite(lib, N, V):
    """a token's NaN stays in its row, a vocabulary row's in its column; masked tokens do not matter"""
    H, hs, W, ws = _head(N, 64, V, 2)
    hs[1], hs[3] = np.nan, np.nan
    z = lib.logits_rows(*_cuda(H, hs, W, ws))
    assert _same(z, row_logits(H, hs, W, ws))
    targets, mask = np.zeros(N, dtype=np.int32), np.ones(N, dtype=np.uint8)
    mask[3] = 0
    logp, lse = lib.token_logprobs_rows(*_cuda(H, hs, W, ws, targets, mask))
    bad = torch.isnan(lse).cpu().numpy()
    assert bad[1] and bad.sum() == 1 and torch.isnan(logp)[1] and float(lse[3]) == 0
    ws[V // 2] = np.nan
    hs[1] = hs[3] = 0.5
    assert _same(lib.logits_rows(*_cuda(H, hs, W, ws)), row_logits(H, hs, W, ws))
    logp, lse = lib.token_logprobs_rows(*_cuda(H, hs, W, ws, targets, mask))                # a distribution with a NaN in it is none
    on = mask != 0
    assert np.isnan(f64(lse))[on].all() and np.isnan(f64(logp))[on].all() and float(lse[3]) == 0


def test_on_another_stream_and_in_a_graph(lib):
    H, hs, W, ws = _head(50, 528, 3000, 6)
    x = torch.randn(50, 528, device="cuda", dtype=torch.bfloat16)
    Wd, wsd, targets = *_cuda(W, ws), torch.arange(50, device="cuda", dtype=torch.int32)

    def step(stream=None):
        q, s = lib.quantise_rows(x, stream=stream)
        return (q, s, lib.logits_rows(q, s, Wd, wsd, stream=stream), *lib.token_logprobs_rows(q, s, Wd, wsd, targets, stream=stream))

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(3):
        x.copy_(torch.randn_like(x))
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), i
