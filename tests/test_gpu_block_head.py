"""The head in 8 bits: quantisation, logits and token log-probabilities against the definitions in 64 bits.

The plain form forms z from exactly the values that the codes and scales stand for, so a tolerance covers sums and the last
rounding only.  u = 2^-24 is half a step of fp32; a random order of d roundings leaves sqrt(d) u of the products' root sum of squares
(rss).  fp32 logits, and every call of up to 64 tokens and 32640 rows of W (more of those fill the chip with tiles), are such sums: 4 (sqrt(d) + 4) u rss
and u of the result.  The 8-bit matrix pipe aligns the products of a block to the largest and drops what lies 2^-14 and further below it: 2^-12 rss allows four of
those at once (a bf16 logit's own rounding is 2^-8 of itself).  A sum of exponentials moves by at most the largest of those errors; the
target's own logit is an fp32 sum."""
import numpy as np
import pytest
import torch

from operator_util import (E4M3, dequantise, e4m3_nearest, e4m3_values, f64, log_softmax_at, make_blocks, quantise, scale_exponents)

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _fp32_sums(N, V):
    return N <= 64 and V <= 32640


def _rng(seed):
    return np.random.default_rng(seed)


# ---- quantisation ----------------------------------------------------------------------------------------------------------------

def _check_quantised(lib, x, block_rows):
    q, scale = lib.quantise_blocks(x, block_rows)
    assert q.dtype == torch.float8_e4m3fn and q.shape == x.shape
    y, e = quantise(f64(x), block_rows)
    got, pad = scale_exponents(scale, e.shape[1])
    assert np.array_equal(got, e) and (pad == 127).all()
    want = e4m3_nearest(np.nan_to_num(y))
    want[np.isnan(y)] = np.nan
    assert np.array_equal(e4m3_values(q), want, equal_nan=True)
    again = lib.quantise_blocks(x, block_rows)
    assert torch.equal(again[0].view(torch.uint8), q.view(torch.uint8)) and torch.equal(again[1].view(torch.uint8), scale.view(torch.uint8))


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("R,C", [(1, 16), (1, 128), (3, 144), (127, 528), (128, 512), (129, 1040), (300, 4096), (5, 2064), (257, 112)])
def test_quantised_exactly(lib, R, C, dtype, block_rows):
    g = _rng(R + C)
    x = g.standard_normal((R, C)) * np.exp(2 * g.standard_normal((1, C)))
    _check_quantised(lib, torch.from_numpy(x).to(dtype).cuda(), block_rows)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantised_borders(lib, block_rows):
    """every value of e4m3 and every midpoint between two, blocks of zeros, of the smallest and the largest numbers, of nothing finite"""
    x = np.zeros((140, 1040), dtype=np.float32)
    mid = (E4M3[1:] + E4M3[:-1]) / 2
    x[0, :127] = E4M3
    x[0, 127] = -448.0
    x[1, 128:254] = mid
    x[1, 254] = 448.0
    x[2, 256:384] = -np.ldexp(E4M3[np.arange(128) % 127], 100)
    x[3, 512:640] = np.float32(1e-45)                                     # below the normal numbers
    x[4, 640:768] = np.float32(3.4028235e38)
    x[5, 768:896] = np.nan
    x[6, 896:1024:2] = np.inf
    x[6, 897:1024:2] = 3.0
    x[7, 1024:] = -np.inf
    x[131] = np.ldexp(np.float32(448.0), -150)
    x[132] = np.nextafter(np.float32(448.0), np.float32(1000))            # just above: the next power
    x[133, :] = 1.0
    x[133, ::128] = 448.0 * 2
    _check_quantised(lib, torch.from_numpy(x).cuda(), block_rows)


# ---- products --------------------------------------------------------------------------------------------------------------------

def _head(N, d, V, seed, spread=0.0):
    g = _rng(seed)
    H = g.standard_normal((N, d)) * np.exp(spread * g.standard_normal((N, d)))
    W = g.standard_normal((V, d)) * d ** -0.5 * np.exp(spread * g.standard_normal((V, 1)))
    return (*make_blocks(H, 1, "cuda"), *make_blocks(W, 128, "cuda"))


def _plain(x):
    H, W = (torch.from_numpy(dequantise(q, s, b)).cuda() for q, s, b in ((x[0], x[1], 1), (x[2], x[3], 128)))
    return (H @ W.T).cpu().numpy(), torch.sqrt((H * H) @ (W * W).T).cpu().numpy()      # products in 64 bits


def _tolerance(z, rss, d, fp32, out_u):
    return out_u * np.abs(z) + ((4 * (d ** 0.5 + 4) * U) if fp32 else 2.0 ** -12) * rss + 1e-40


TOKENS = [1, 15, 16, 17, 32, 33, 48, 64, 65, 127, 128, 129, 257]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("i,N", enumerate(TOKENS))
def test_logits(lib, i, N, dtype):
    for j, (d, V) in enumerate([(16, 1), (128, 33), (144, 300), (528, 129), (1040, 257), (2064, 1000), (4096, 64)]):
        x = _head(N, d, V, 100 * i + j, spread=j % 2)
        z, rss = _plain(x)
        out = torch.full((N + 2, V), 7.0, dtype=dtype, device="cuda")     # what lies before and behind stays
        got = lib.logits_blocks(*x, out=out[1:N + 1]) if V % 8 == 0 else lib.logits_blocks(*x, dtype=dtype)
        assert got.shape == (N, V) and got.dtype == dtype
        assert (out[0] == 7).all() and (out[N + 1] == 7).all()
        tol = _tolerance(z, rss, d, dtype == torch.float32 or _fp32_sums(N, V), U if dtype == torch.float32 else 2.0 ** -8)
        assert (np.abs(f64(got) - z) <= tol).all(), (N, d, V)
        assert torch.equal(got, lib.logits_blocks(*x, dtype=dtype))        # the same call gives the same bits


@pytest.mark.parametrize("N,d,V,dtype", [(300, 1168, 20001, torch.bfloat16), (70, 2048, 33000, torch.bfloat16), (1100, 272, 12345, torch.bfloat16),
                                         (64, 4624, 10000, torch.float32), (150, 656, 20011, torch.float32), (2000, 128, 8200, torch.bfloat16),
                                         (300, 1024, 8000, torch.float32), (300, 1024, 8000, torch.bfloat16), (3000, 144, 500, torch.bfloat16),
                                         (430, 144, 32969, torch.bfloat16), (530, 144, 26309, torch.bfloat16),
                                         (40, 272, 33000, torch.float32), (3, 144, 40001, torch.float32), (64, 1040, 32641, torch.bfloat16)])
def test_logits_of_many_tiles(lib, N, d, V, dtype):
    """more tiles than workgroups, turned slabs (few columns of tiles), every kernel's last tile in both directions, the last rows of W on smaller tiles
    (two kinds)"""
    x = _head(N, d, V, N)
    z, rss = _plain(x)
    tol = _tolerance(z, rss, d, dtype == torch.float32 or _fp32_sums(N, V), U if dtype == torch.float32 else 2.0 ** -8)
    assert (np.abs(f64(lib.logits_blocks(*x, dtype=dtype)) - z) <= tol).all()


def test_scales_of_every_block_and_row_count(lib):
    """scales that differ by up to 2^30 from block to block, so that one taken for another is far outside any tolerance"""
    for N, V, d in ((5, 400, 1040), (100, 400, 1552), (300, 700, 2064)):
        g = _rng(N)
        He, We = g.integers(-15, 16, (N, -(-d // 128))), g.integers(-15, 16, (-(-V // 128), -(-d // 128)))
        H = g.standard_normal((N, d)) * np.exp2(np.repeat(He, 128, 1)[:, :d])
        W = g.standard_normal((V, d)) * np.exp2(np.repeat(np.repeat(We, 128, 0)[:V], 128, 1)[:, :d])
        x = (*make_blocks(H, 1, "cuda"), *make_blocks(W, 128, "cuda"))
        z, rss = _plain(x)
        for dtype in (torch.float32, torch.bfloat16):
            tol = _tolerance(z, rss, d, dtype == torch.float32 or _fp32_sums(N, V), U if dtype == torch.float32 else 2.0 ** -8)
            assert (np.abs(f64(lib.logits_blocks(*x, dtype=dtype)) - z) <= tol).all()


def _check_logprobs(lib, x, targets, mask, d, V, **kw):
    N = x[0].shape[0]
    z, rss = _plain(x)
    t = torch.from_numpy(targets.astype(np.int32)).cuda()
    m = None if mask is None else torch.from_numpy(mask.astype(np.uint8)).cuda()
    logp, lse = lib.token_logprobs_blocks(*x, t, m, **kw)
    active = (targets >= 0) & (targets < V) & (True if mask is None else mask != 0)
    assert (f64(logp)[~active] == 0).all() and (f64(lse)[~active] == 0).all()
    want_logp, want_lse = log_softmax_at(z[active], targets[active])
    fp32 = 4 * (d ** 0.5 + 4) * U * rss[active].max(axis=1, initial=0)
    pipe = fp32 if _fp32_sums(N, V) else 2.0 ** -12 * rss[active].max(axis=1, initial=0)
    last = 16 * U * (np.abs(want_lse) + np.abs(want_logp) + 8)             # exp, log and the merge of the tiles' sums
    assert (np.abs(f64(lse)[active] - want_lse) <= pipe + last).all()
    assert (np.abs(f64(logp)[active] - want_logp) <= pipe + fp32 + last).all()
    return logp, lse


@pytest.mark.parametrize("N", TOKENS)
def test_log_probabilities(lib, N):
    for j, (d, V) in enumerate([(16, 1), (128, 33), (528, 1000), (1040, 257), (4096, 640)]):
        x, g = _head(N, d, V, N + j), _rng(N * j)
        targets = g.integers(0, V, N)
        a = _check_logprobs(lib, x, targets, None, d, V)
        b = _check_logprobs(lib, x, targets, None, d, V)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        mask = g.integers(0, 2, N)
        targets[:: 5] = -1
        targets[1:: 7] = V
        c = _check_logprobs(lib, x, targets, mask, d, V)
        _check_logprobs(lib, x, targets, np.zeros(N), d, V)
        # an active row does not depend on which others are, up to the order of sums; an all-active call gives its bits for up to 64 tokens
        if _fp32_sums(N, V):
            on = (mask != 0) & (targets >= 0) & (targets < V)
            assert np.array_equal(f64(c[1])[on], f64(a[1])[on])


@pytest.mark.parametrize("N,d,V", [(300, 1168, 20001), (70, 2048, 33000), (1100, 272, 12345), (64, 4624, 10000), (40, 512, 128256),
                                   (300, 1024, 8000), (348, 528, 5000), (3000, 144, 500)])      # small tiles, many of them
def test_log_probabilities_of_many_tiles(lib, N, d, V):
    x, g = _head(N, d, V, N), _rng(N)
    _check_logprobs(lib, x, g.integers(0, V, N), g.integers(0, 4, N), d, V)


def test_rows_that_are_masked_do_not_reach_the_others(lib):
    for N in (40, 200):
        x = _head(N, 528, 700, N)
        targets, mask = _rng(N).integers(0, 700, N), np.ones(N)
        mask[::3] = 0
        good = _check_logprobs(lib, x, targets, mask, 528, 700)
        x[0].view(torch.uint8)[::3] = 0x7F                                 # NaN in every masked row
        t, m = torch.from_numpy(targets.astype(np.int32)).cuda(), torch.from_numpy(mask.astype(np.uint8)).cuda()
        bad = lib.token_logprobs_blocks(*x, t, m)
        assert torch.equal(good[0], bad[0]) and torch.equal(good[1], bad[1])


def test_values_that_are_not_finite_stay_in_their_row_and_column(lib):
    for N in (40, 200):
        for dtype in (torch.float32, torch.bfloat16):
            x = _head(N, 528, 700, N)
            x[0].view(torch.uint8)[3, 100] = 0x7F
            x[2].view(torch.uint8)[650, 520] = 0xFF
            z = torch.isnan(lib.logits_blocks(*x, dtype=dtype))
            want = torch.zeros_like(z)
            want[3] = True
            want[:, 650] = True
            assert torch.equal(z, want)


def test_scales_at_the_ends_of_their_range(lib):
    """products of entries below the normal numbers with ones near the largest"""
    for N in (20, 100):
        H, W = np.full((N, 256), 448.0 * 2.0 ** 100), np.full((300, 256), 448.0 * 2.0 ** -127)
        H[:, 128:] = 0
        x = (*make_blocks(H, 1, "cuda"), *make_blocks(W, 128, "cuda"))
        z, _ = _plain(x)
        assert np.allclose(f64(lib.logits_blocks(*x)), z, rtol=1e-6, atol=0)


def test_replayed_from_a_graph(lib):
    N, d, V = 150, 528, 3000
    variants = [_head(N, d, V, s) for s in range(3)]
    targets = torch.randint(0, V, (N,), device="cuda").int()
    mask = (torch.rand(N, device="cuda") < 0.7).to(torch.uint8)
    H = torch.randn(N, d, device="cuda", dtype=torch.bfloat16)
    few = 20
    x = [t.view(torch.uint8).clone().view(t.dtype) for t in variants[0]]
    ws = [torch.empty(lib.logprobs_blocks_workspace_bytes(n, V), dtype=torch.uint8, device="cuda") for n in (N, few)]

    def calls():
        q, s = lib.quantise_blocks(H, 1)
        return [lib.logits_blocks(*x, dtype=torch.bfloat16), *lib.token_logprobs_blocks(*x, targets, mask, ws=ws[0]), lib.logits_blocks(q, s, *x[2:]),
                *lib.token_logprobs_blocks(x[0][:few], x[1][:, :few].contiguous(), *x[2:], targets[:few], mask[:few], ws=ws[1])]

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = calls()
    torch.cuda.synchronize()
    for rep, i in enumerate((1, 2, 0, 1)):
        for a, b in zip(x, variants[i]):
            a.view(torch.uint8).copy_(b.view(torch.uint8))
        H.normal_()
        for t in got:
            t.fill_(float("nan"))
        for w in ws:
            w.fill_(0xA5 if rep % 2 else 0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, calls()):
            assert torch.equal(a, b), rep


def test_arguments_are_checked(lib):
    H, Hs, W, Ws = _head(10, 144, 300, 1)
    t = torch.zeros(10, dtype=torch.int32, device="cuda")
    for bad in ((H, Hs, W, Hs), (H, Ws, W, Ws), (H.float(), Hs, W, Ws), (H, Hs.view(torch.uint8), W, Ws), (H, Hs, W[:, :128], Ws), (H[:, ::2], Hs, W, Ws),
                (H, Hs[:, :9], W, Ws), (H[0], Hs, W, Ws), (H.cpu(), Hs, W, Ws), (H, Hs.cpu(), W, Ws), (H, Hs, W, Ws.transpose(0, 1))):
        with pytest.raises(lib.LlamarlError):
            lib.logits_blocks(*bad)
        with pytest.raises(lib.LlamarlError):
            lib.token_logprobs_blocks(*bad, t)
    for bad in (dict(out=torch.empty(10, 299, device="cuda")), dict(out=torch.empty(300, 10, device="cuda").T), dict(dtype=torch.float16),
                dict(out=torch.empty(10, 300))):
        with pytest.raises(lib.LlamarlError):
            lib.logits_blocks(H, Hs, W, Ws, **bad)
    for bad in (dict(targets=t[:9]), dict(targets=t.long()), dict(targets=t, mask=t), dict(targets=t, mask=t[:9].to(torch.uint8)),
                dict(targets=t, ws=torch.empty(64, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(lib.LlamarlError):
            lib.token_logprobs_blocks(H, Hs, W, Ws, **bad)
    x = torch.zeros(4, 32, device="cuda")
    for bad in ((x, 2), (x[:, ::2], 1), (x.T, 1), (x.half(), 1), (x[0], 1), (x[:, :8].contiguous(), 1)):
        with pytest.raises(lib.LlamarlError):
            lib.quantise_blocks(*bad)


def test_on_a_stream_of_its_own(lib):
    side = torch.cuda.Stream()
    for N in (30, 300):
        H, Hs, W, Ws = _head(N, 528, 1000, N)
        t = torch.zeros(N, dtype=torch.int32, device="cuda")
        x = torch.randn(N, 528, device="cuda")
        torch.cuda.synchronize()
        got = [*lib.quantise_blocks(x, 1, stream=side), lib.logits_blocks(H, Hs, W, Ws, stream=side), *lib.token_logprobs_blocks(H, Hs, W, Ws, t, stream=side)]
        side.synchronize()
        want = [*lib.quantise_blocks(x, 1), lib.logits_blocks(H, Hs, W, Ws), *lib.token_logprobs_blocks(H, Hs, W, Ws, t)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_two_streams_at_once(lib):
    """calls whose workspaces and outputs are their own: as one after the other"""
    calls = []
    for i, N in enumerate((700, 40, 650, 30)):
        x = _head(N, 528, 5000, 40 + i)
        t = torch.from_numpy(_rng(i).integers(0, 5000, N).astype(np.int32)).cuda()
        calls.append((x, t, lib.token_logprobs_blocks(*x, t), lib.logits_blocks(*x)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for turn in range(3):
        for i, (x, t, _, _) in enumerate(calls):
            with torch.cuda.stream(streams[i % 2]):
                got.append((i, lib.token_logprobs_blocks(*x, t), lib.logits_blocks(*x)))
    torch.cuda.synchronize()
    for i, (logp, lse), z in got:
        assert torch.equal(logp, calls[i][2][0]) and torch.equal(lse, calls[i][2][1]) and torch.equal(z, calls[i][3])


@pytest.mark.parametrize("N", [5, 40, 130, 700])
def test_scratch_is_written_before_it_is_read(lib, N):
    x, g = _head(N, 528, 5000, N), _rng(N)
    t, m = torch.from_numpy(g.integers(0, 5000, N).astype(np.int32)).cuda(), torch.from_numpy(g.integers(0, 2, N).astype(np.uint8)).cuda()
    want = lib.token_logprobs_blocks(*x, t, m)
    size = lib.logprobs_blocks_workspace_bytes(N, 5000)
    for fill in (0xFF, 0x7F, 0):
        ws = torch.full((size + 64,), fill, dtype=torch.uint8, device="cuda")
        got = lib.token_logprobs_blocks(*x, t, m, ws=ws[:size])
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and bool((ws[size:] == fill).all())
