"""Plain forms of the optimiser step and of the 8-bit head, in 64 bits (numpy and torch on the CPU), shared by the operators' tests."""
import math

import numpy as np
import torch

BLOCK = 128
E4M3_MAX = 448.0
# the values of e4m3 (OCP): sign, four exponent bits (bias 7), three of mantissa; 0x7f is NaN
E4M3 = np.array([(1 + (c & 7) / 8.0) * 2.0 ** ((c >> 3) - 7) if c >> 3 else (c & 7) * 2.0 ** -9 for c in range(127)])


def f64(t):
    return t.detach().cpu().double().numpy() if t.dtype not in (torch.float8_e4m3fn, torch.float8_e8m0fnu) else \
        t.detach().cpu().view(torch.uint8).numpy()


def e4m3_values(q):
    """float8_e4m3fn tensor -> float64, by the definition of the format"""
    c = f64(q).astype(np.int64)
    mag = np.append(E4M3, np.nan)[c & 127]
    return np.where(c & 128, -mag, mag)


def e4m3_nearest(x):
    """float64 in [-448, 448] -> the nearest e4m3 value, ties to the even code"""
    a = np.abs(x)
    hi = np.clip(np.searchsorted(E4M3, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    below, above = a - E4M3[lo], E4M3[hi] - a
    code = np.where(below < above, lo, np.where(above < below, hi, np.where(lo % 2 == 0, lo, hi)))
    return np.sign(x) * E4M3[code]


def rounding_bits(n, step, place):
    """the 16 random bits of each of a tensor's n entries"""
    i = np.arange(n, dtype=np.uint64)
    low = np.uint64(0xFFFFFFFF)
    x = (i // 2 + np.uint64(step % 2 ** 32 * 0x9E3779B9 % 2 ** 32) + np.uint64(place * 0xB504F333 % 2 ** 32)) & low
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0xDDB3D743)) & low
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0x8F1BBCDD)) & low
    x ^= x >> np.uint64(16)
    return np.where(i % 2 == 1, x >> np.uint64(16), x & np.uint64(0xFFFF)).astype(np.int64)


def blocks_of(x):
    """[n] -> [ceil(n / 128), 128], zeros behind"""
    n = x.size
    return np.pad(x, (0, -n % BLOCK)).reshape(-1, BLOCK)


def adamw(p, g, m, v, lr, t, b1, b2, eps, wd, scale=1.0):
    """float64 arrays -> new (p, m, v)"""
    g = g * scale
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    update = (m / (1 - b1 ** t)) / (np.sqrt(v / (1 - b2 ** t)) + eps)
    return p - lr * (wd * p + update), m, v


def quantise(x, block_rows):
    """float64 [R, C] -> (values in units of the block's scale, not rounded; exponent table [ceil(R / block_rows), ceil(C / 128)])"""
    R, C = x.shape
    Rb, Cb = -(-R // block_rows), -(-C // BLOCK)
    y, e = np.empty_like(x), np.zeros((Rb, Cb), dtype=np.int64)
    for r in range(Rb):
        for c in range(Cb):
            at = (slice(r * block_rows, (r + 1) * block_rows), slice(c * BLOCK, (c + 1) * BLOCK))
            b = np.where(np.isfinite(x[at]), np.abs(x[at]), 0.0)
            top = b.max()
            if top > 0:
                e[r, c] = max(math.frexp(top / E4M3_MAX)[1] - (math.frexp(top / E4M3_MAX)[0] == 0.5), -127)
            y[at] = np.where(np.isfinite(x[at]), np.ldexp(x[at], -e[r, c]), np.nan)
    return y, e


def scale_exponents(scale, blocks):
    """float8_e8m0fnu [G, R, 4] -> exponents [R, blocks], and the bytes past them"""
    s = f64(scale).astype(np.int64).transpose(1, 0, 2).reshape(scale.shape[1], -1)
    return s[:, :blocks] - 127, s[:, blocks:]


def dequantise(q, scale, block_rows):
    """what (q, scale) stand for, float64"""
    R, C = q.shape
    e, _ = scale_exponents(scale, -(-C // BLOCK))
    e = np.repeat(np.repeat(e, block_rows, axis=0)[:R], BLOCK, axis=1)[:, :C]
    return np.ldexp(e4m3_values(q), e)


def make_blocks(x, block_rows, device):
    """float64 [R, C] quantised by the plain form, as tensors on `device`"""
    y, e = quantise(x, block_rows)
    v = e4m3_nearest(y)
    code = np.searchsorted(E4M3, np.abs(v)) | np.where(np.signbit(v), 128, 0)
    q = torch.from_numpy(code.astype(np.uint8)).to(device).view(torch.float8_e4m3fn)
    Cb = e.shape[1]
    s = np.full((e.shape[0], -(-Cb // 4) * 4), 127, dtype=np.uint8)
    s[:, :Cb] = e + 127
    s = np.ascontiguousarray(s.reshape(e.shape[0], -1, 4).transpose(1, 0, 2))
    return q, torch.from_numpy(s).to(device).view(torch.float8_e8m0fnu)


def log_softmax_at(z, targets):
    top = z.max(axis=1)
    lse = np.log(np.exp(z - top[:, None]).sum(axis=1)) + top
    return z[np.arange(z.shape[0]), targets] - lse, lse
