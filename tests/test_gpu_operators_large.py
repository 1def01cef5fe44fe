"""Arrays of more than 2^31 entries: what lies at their end comes out as the same values do in a small call."""
import pytest
import torch

from operator_util import dequantise, f64

pytestmark = pytest.mark.gpu
BIG = 2 ** 31


@pytest.fixture(autouse=True)
def _room():
    yield
    torch.cuda.empty_cache()


def _random_codes(rows, cols, seed):
    """finite e4m3 codes, made in place"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    q = torch.randint(0, 256, (rows, cols), generator=g, device="cuda", dtype=torch.uint8)
    q.bitwise_and_(0xB7)                                                   # exponents up to 6: magnitudes below 1, no NaN
    return q.view(torch.float8_e4m3fn)


def _scales(cols, rows, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(124, 130, (-(-cols // 512), rows, 4), generator=g, device="cuda", dtype=torch.uint8).view(torch.float8_e8m0fnu)


def _some(scale, rows):
    return scale.view(torch.uint8)[:, rows].contiguous().view(scale.dtype)


@pytest.mark.parametrize("bits", [8, 32])
def test_adamw_and_norm(lib, bits):
    n, tail = BIG + 128 * 40 + 77, 128 * 30 + 77
    dt = torch.bfloat16
    p, g = torch.zeros(n, dtype=dt, device="cuda"), torch.zeros(n, dtype=dt, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    p[-tail:] = torch.randn(tail, generator=gen, device="cuda").to(dt)
    g[-tail:] = torch.randn(tail, generator=gen, device="cuda").to(dt)
    norm, scale = lib.grad_norm([g], 1.0)
    want = g[-tail:].double().norm().item()
    assert abs(float(norm) / want - 1) < 1e-6
    small_p, small_g = p[-tail:].clone(), g[-tail:].clone()

    def states(k):
        if bits == 32:
            return [torch.zeros(k, device="cuda") for _ in range(2)] + [None, None]
        return [torch.zeros(k, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)] + \
               [torch.zeros(-(-k // 128), device="cuda") for _ in range(2)]

    a, b = states(n), states(tail)
    for x, y, s in ((p, g, a), (small_p, small_g, b)):
        lib.adamw_step([x], [y], [s[0]], [s[1]], 1e-2, 1, exp_avg_scales=[s[2]], exp_avg_sq_scales=[s[3]], grad_scale=scale)
    assert torch.equal(p[-tail:], small_p)
    assert torch.equal(a[0].view(torch.uint8)[-tail * (bits // 8):], b[0].view(torch.uint8))         # m; sqrt(v) is rounded by its place in 8 bits
    if bits == 8:
        assert torch.equal(a[2][-len(b[2]):], b[2]) and torch.equal(a[3][-len(b[3]):], b[3])
    assert not p[:-tail].any()


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quantise(lib, block_rows):
    R, C, tail = 128 * 8200 + 3, 2064, 128 + 3
    assert R * C > BIG
    x = torch.zeros(R, C, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(2)
    x[-tail:] = torch.randn(tail, C, generator=gen, device="cuda").to(x.dtype)
    q, s = lib.quantise_blocks(x, block_rows)
    sq, ss = lib.quantise_blocks(x[-tail:].contiguous(), block_rows)
    assert torch.equal(q[-tail:].view(torch.uint8), sq.view(torch.uint8)) and not q[:-tail].view(torch.uint8).any()
    assert torch.equal(s.view(torch.uint8)[:, -ss.shape[1]:], ss.view(torch.uint8))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_logits(lib, dtype):
    N, d, V = 16800, 32, 128256
    assert N * V > BIG
    x = _random_codes(N, d, 3), _scales(d, N, 4), _random_codes(V, d, 5), _scales(d, -(-V // 128), 6)
    z = lib.logits_blocks(*x, dtype=dtype)
    for rows in (slice(0, 2), slice(N // 2, N // 2 + 2), slice(N - 3, N)):
        H = torch.from_numpy(dequantise(x[0][rows], _some(x[1], rows), 1))
        want = H @ torch.from_numpy(dequantise(x[2], x[3], 128)).T
        rss = ((H * H) @ (torch.from_numpy(dequantise(x[2], x[3], 128)) ** 2).T).sqrt()
        got = torch.from_numpy(f64(z[rows]))
        # half a step of the result; sums of 32 products: 4 (sqrt(32) + 4) 2^-24 rss in fp32, 2^-12 rss on the 8-bit pipe
        tol = want.abs() * 2.0 ** -24 + rss * 2.4e-6 if dtype == torch.float32 else want.abs() * 2.0 ** -8 + rss * 2.0 ** -12
        assert ((got - want).abs() <= tol).all()


@pytest.mark.parametrize("N", [3, 40, 70])
def test_weights(lib, N):
    d, V = 4112, 128 * 4096 + 1000
    assert d * V > BIG
    H, Hs, W, Ws = _random_codes(N, d, 7), _scales(d, N, 8), _random_codes(V, d, 9), _scales(d, -(-V // 128), 10)
    z, tail = lib.logits_blocks(H, Hs, W, Ws), 1000
    targets = torch.full((N,), V - 1, dtype=torch.int32, device="cuda")
    targets[0] = 5
    logp, lse = lib.token_logprobs_blocks(H, Hs, W, Ws, targets)
    last = W[-tail:], _some(Ws, slice(-8, None))
    small = lib.logits_blocks(H, Hs, *last)
    Hd = torch.from_numpy(dequantise(H, Hs, 1))
    rss = ((Hd * Hd) @ (torch.from_numpy(dequantise(*last, 128)) ** 2).T).sqrt()
    assert ((z[:, -tail:] - small).cpu().double().abs() <= 8 * (d ** 0.5 + 4) * 2.0 ** -24 * rss).all()      # two fp32 sums, in orders of their own
    # an lse is off by 2^-12 of a row's rss at most, which entries of W below 4 (codes below 1, scales up to 4) bound by 4 |h|
    pipe = (2.0 ** -10 * Hd.norm(dim=1)).cuda()
    want = torch.logsumexp(z.double(), 1)
    assert ((lse.double() - want).abs() <= pipe + 1e-6 * want.abs()).all()
    got = z.double()[torch.arange(N, device="cuda"), targets.long()] - want
    assert ((logp.double() - got).abs() <= 2 * pipe + 1e-6 * (want.abs() + got.abs())).all()
