"""Plain forms, in 64 bits (numpy), of the norm, of the head in 8-bit integers and of the verification of drafted tokens."""
import math

import numpy as np

U = 2.0 ** -24                    # half a step of fp32
HALF = {"torch.float32": 2.0 ** -24, "torch.bfloat16": 2.0 ** -8}


def rms(s, w, eps):
    """float64 s [N, d], w [d] -> (h, n = s rstd, rstd [N, 1])"""
    r = 1.0 / np.sqrt((s * s).mean(axis=1, keepdims=True) + eps)
    return s * r * w, s * r, r


def rms_bwd(dh, s, w, eps, dsum=None):
    """gradients of sum(dh * h) + sum(dsum * s): (dx, dw)"""
    _, n, r = rms(s, w, eps)
    g = dh * w
    dx = r * (g - n * (g * n).mean(axis=1, keepdims=True))
    return dx if dsum is None else dx + dsum, (dh * n).sum(axis=0)


def quantise_rows(x):
    """float32 [R, C] -> (int8, float32 [R]), every operation in fp32"""
    x = np.asarray(x, dtype=np.float32)
    with np.errstate(all="ignore"):
        top = np.abs(x).max(axis=1)
        bad = ~np.isfinite(x).all(axis=1)
        scale = np.where(top < np.float32(2.0 ** -100), np.float32(0), top / np.float32(127)).astype(np.float32)
        scale = np.where(bad, np.float32(np.nan), scale)
        q = np.rint(x / np.where(scale > 0, scale, np.float32(1))[:, None])
        q = np.where((scale > 0)[:, None], q, 0)
    return q.astype(np.int8), scale


def row_logits(H, hs, W, ws):
    """the product's sum exactly, then its three fp32 roundings"""
    with np.errstate(invalid="ignore", over="ignore"):
        z = (H.astype(np.float64) @ W.astype(np.float64).T).astype(np.float32)
        return z * ws[None, :] * hs[:, None]


def _distribution(row, T):
    """None where there is none"""
    row = row.astype(np.float64)
    if not (T >= 0 and math.isfinite(T)) or np.isnan(row).any() or (row == np.inf).any() or (row == -np.inf).all():
        return None
    p = np.zeros_like(row)
    if T == 0:
        p[int(np.argmax(row))] = 1.0                                      # the first of equal ones
        return p
    e = np.exp((row - row.max()) / T)
    return e / e.sum()


def verify(logits, drafts, u, draft_logits=None, lens=None, temps=None):
    """arrays -> (tokens, accepted, logp), one sequence after the other"""
    B, K1, V = logits.shape
    K = K1 - 1
    tokens, accepted, logp = np.full((B, K1), -1, dtype=np.int64), np.zeros(B, dtype=np.int64), np.zeros((B, K1))
    for b in range(B):
        T = 1.0 if temps is None else float(temps[b])
        n = K if lens is None else min(max(int(lens[b]), 0), K)
        for i in range(n + 1):
            p = _distribution(logits[b, i], T)
            r = p
            if i < n:
                x = int(drafts[b, i])
                inside = 0 <= x < V
                if draft_logits is None or T == 0:
                    q = np.zeros(V)
                    if inside:
                        q[x] = 1.0
                else:
                    q = _distribution(draft_logits[b, i], T)
                if p is not None and q is not None:
                    given = float(u[b, i])
                    if inside and (0.0 if given < 0 else given) * q[x] < p[x]:
                        tokens[b, i], logp[b, i] = x, (0.0 if T == 0 else math.log(p[x]))
                        continue
                    r = np.maximum(p - q, 0.0)
                    r = r if r.sum() > 2.0 ** -40 else p                   # less is the rounding of p and q
                else:
                    r = None
            accepted[b] = i
            if r is None:
                logp[b, i] = np.nan
            else:
                last = float(u[b, K])
                last = 0.0 if not last > 0 else min(last, 1 - 2.0 ** -24)
                c = np.cumsum(r)
                y = int(np.searchsorted(c, last * c[-1], side="right"))
                tokens[b, i], logp[b, i] = y, (0.0 if T == 0 else math.log(p[y]))
            break
    return tokens, accepted, logp
