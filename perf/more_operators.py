"""Measured operators: the norm in front of the head, a head in 8-bit integers, and the verification of drafted tokens.

A case is a dict of plain values; `kind` says which pass it makes:

  norm      rms_norm of the residual stream (with the residual's addition or without) and rms_norm_bwd: a training step's share
  norm8     the same norm for a generator, its output in 8 bits: e4m3 in blocks of 128 or int8 with a scale for each token
  logits    hidden states quantised to int8 and multiplied with an int8 head (a scale for each token and each vocabulary row)
  logprobs  the log-probabilities of given tokens under that head (the generator's mu), without logits in memory
  verify    drafted tokens accepted or replaced under the target's logits from given random numbers, with their log-probabilities

`run` makes the framework's calls where `own` is true, and the same from elementary torch operations elsewhere.  Sizes are those of
the benchmark workloads' heads (tiny, Llama-3-8B, one of eight ranks of 70B), of the tests and generic ones.
"""
import math

import torch

own = False

DEV = "cuda"
FULL_V = 128256
BLOCK = 128
E4M3_MAX = 448.0
INT8_MAX = 127.0
TINY = 2.0 ** -100                # a row below this is zeros in int8
EPS = 1e-5


def listed():
    return [
        # a unit-test sized fp32 model's final norm, no residual: launch latency counts
        dict(name="norm_small_odd_f32", kind="norm", N=333, d=520, dtype="f32", residual=False),
        # the final norm of a trainer batch at the 8B shape, forward and backward
        dict(name="norm_8b", kind="norm", N=16384, d=4096, dtype="bf16", residual=True),
        # one decoding step of one sequence in front of an int8 head
        dict(name="norm8_rows_one_token", kind="norm8", N=1, d=4096, dtype="bf16", residual=True, out="rows"),
        # a prompt in front of a head in 8-bit blocks
        dict(name="norm8_blocks_prompt", kind="norm8", N=1900, d=8192, dtype="bf16", residual=True, out="blocks"),
        # one decoding step of one sequence at the 8B head: the weights' bytes are the time
        dict(name="logits_8b_one_token", kind="logits", N=1, d=4096, V=FULL_V, out="f32"),
        # 48 positions (eight sequences with five drafts each) on one of eight ranks of the 70B head
        dict(name="logits_70b_rank_48", kind="logits", N=48, d=8192, V=16032, out="f32"),
        # a prompt's logits under a ~1B-class head
        dict(name="logits_1b_prompt", kind="logits", N=1900, d=2048, V=33001, out="bf16"),
        # a debugging run: no size a multiple of a tile
        dict(name="logprobs_small_odd", kind="logprobs", B=3, T=347, len_lo=40, d=528, V=5003),
        # mu of a trainer batch at the 8B shape
        dict(name="logprobs_8b", kind="logprobs", B=8, T=2048, len_lo=256, d=4096, V=FULL_V),
        # drafts copied from the prompt (no draft distribution), a small vocabulary, sequences of different numbers of drafts
        dict(name="verify_copied_small", kind="verify", B=7, K=3, V=5003, dtype="f32", drafts="copied", ragged=True, greedy=0.3),
        # one sequence with four drafts of a smaller model: latency counts
        dict(name="verify_one", kind="verify", B=1, K=4, V=FULL_V, dtype="f32", drafts="model", ragged=False, greedy=0.0),
        # a generator's batch, five drafts each
        dict(name="verify_batch", kind="verify", B=64, K=5, V=FULL_V, dtype="bf16", drafts="model", ragged=True, greedy=0.1),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm8", "logits", "logits", "logprobs", "verify", "verify"])
    if kind in ("norm", "norm8"):
        d = (8 if kind == "norm" else 16) * _log_int(rng, 4, 1024 if kind == "norm" else 512)
        dtype = rng.choice(["bf16", "f32"])
        case = dict(kind=kind, N=_log_int(rng, 1, 16384 * 4096 // 2 // d), d=d, dtype=dtype, residual=rng.random() < 0.7)
        if kind == "norm8":
            case["out"] = rng.choice(["rows", "blocks"])
        return case
    if kind == "verify":
        while True:
            B, K = _log_int(rng, 1, 256), rng.choice([0, 1, 2, 3, 4, 5, 8])
            V = FULL_V if rng.random() < 0.3 else _log_int(rng, 100, FULL_V)
            if B * (2 * K + 1) * V <= 64 * 11 * FULL_V:
                break
        return dict(kind=kind, B=B, K=K, V=V, dtype=rng.choice(["bf16", "f32"]) if B * (2 * K + 1) * V <= 32 * 11 * FULL_V else "bf16",
                    drafts=rng.choice(["model", "copied"]), ragged=rng.random() < 0.5, greedy=rng.choice([0.0, 0.2, 1.0]))
    d = 16 * _log_int(rng, 8, 512)
    while True:
        V = FULL_V if rng.random() < 0.3 else _log_int(rng, 1000, FULL_V)
        N = _log_int(rng, 1, 4096 if kind == "logits" else 16384)
        if N * V * d <= 4e12 and N * V <= 3e8:
            break
    if kind == "logits":
        return dict(kind=kind, N=N, d=d, V=V, out=rng.choice(["bf16", "f32"]))
    B = min(N, rng.choice([1, 2, 3, 4, 8]))
    T = N // B
    return dict(kind=kind, B=B, T=T, len_lo=max(1, T // rng.choice([1, 2, 8])), d=d, V=V)


# ---- inputs -------------------------------------------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * seed + 17)
    return g


def _rand(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _mask(g, B, T, len_lo):
    lens = len_lo + torch.floor(torch.rand(B, generator=g, device=DEV) * (T - len_lo + 1)).long().clamp_(max=T - len_lo)
    return (torch.arange(T, device=DEV)[None, :] < lens[:, None]).to(torch.uint8).contiguous()


def _prepare_norm(case, g):
    N, d, dt = case["N"], case["d"], _dtype(case["dtype"])
    size = torch.exp(0.5 * _rand(g, 1, d))                                # channels of different size, some of them outliers
    st = dict(case=case, x=(_rand(g, N, d) * size).to(dt), weight=(1 + 0.2 * _rand(g, d)).to(dt), residual=None, dsum=None)
    if case["residual"]:
        st["residual"] = (2 * _rand(g, N, d) * size).to(dt)
    if case["kind"] == "norm":
        st["dh"] = (1e-3 * _rand(g, N, d)).to(dt)
        if case["residual"]:
            st["dsum"] = (1e-3 * _rand(g, N, d)).to(dt)                   # what the layers behind send back along the stream
    return st


def _prepare_verify(case, g):
    B, K, V, dt = case["B"], case["K"], case["V"], _dtype(case["dtype"])
    logits = torch.empty(B, K + 1, V, dtype=dt, device=DEV)
    draft_logits = torch.empty(B, K, V, dtype=dt, device=DEV) if case["drafts"] == "model" and K > 0 else None
    drafts = torch.zeros(B, K, dtype=torch.int32, device=DEV)
    temperature = 0.6 + 0.6 * torch.rand(B, generator=g, device=DEV)
    temperature = torch.where(torch.rand(B, generator=g, device=DEV) < case["greedy"], torch.zeros_like(temperature), temperature)
    t = torch.where(temperature > 0, temperature, torch.full_like(temperature, 0.05))[:, None]
    for i in range(K + 1):
        z = 2.5 * _rand(g, B, V)
        logits[:, i] = z.to(dt)
        if i < K:
            y = z + 0.7 * _rand(g, B, V) if draft_logits is not None else z + 1.5 * _rand(g, B, V)
            if draft_logits is not None:
                draft_logits[:, i] = y.to(dt)
                y = draft_logits[:, i].float()
            u = torch.rand(B, V, generator=g, device=DEV).clamp_(min=1e-20)
            drafts[:, i] = (y / t - torch.log(-torch.log(u))).argmax(dim=1).to(torch.int32)
    lens = torch.full((B,), K, dtype=torch.int32, device=DEV)
    if case["ragged"]:
        lens = torch.floor(torch.rand(B, generator=g, device=DEV) * (K + 1)).to(torch.int32).clamp_(max=K)
    return dict(case=case, logits=logits, draft_logits=draft_logits, drafts=drafts, lens=lens, temperature=temperature,
                uniforms=torch.rand(B, K + 1, generator=g, device=DEV))


def prepare(case, seed):
    g = _gen(seed)
    if case["kind"] in ("norm", "norm8"):
        return _prepare_norm(case, g)
    if case["kind"] == "verify":
        return _prepare_verify(case, g)
    d = case["d"]
    N = case["N"] if case["kind"] == "logits" else case["B"] * case["T"]
    H = _rand(g, N, d).to(torch.bfloat16)                                 # after the final norm
    Wq, Ws = _plain_quantise_rows((_rand(g, case["V"], d) * d ** -0.5).to(torch.bfloat16).float())
    st = dict(case=case, H=H, Wq=Wq, Ws=Ws)
    if case["kind"] == "logprobs":
        st["mask"] = _mask(g, case["B"], case["T"], case["len_lo"])
        st["targets"] = torch.randint(0, case["V"], (N,), generator=g, device=DEV).to(torch.int32)
    return st


# ---- plain forms ----------------------------------------------------------------------------------------------------------

def _plain_quantise_rows(x):
    """x [R, C] -> (int8 [R, C], float32 [R]): scale = largest magnitude / 127, quotients in fp32, to nearest even"""
    top = x.abs().amax(dim=1)
    scale = torch.where(top < TINY, torch.zeros_like(top), top / torch.full_like(top, INT8_MAX))      # a division, no reciprocal
    q = torch.where(scale[:, None] > 0, x / scale[:, None], torch.zeros_like(x))
    return q.round().clamp(-INT8_MAX, INT8_MAX).to(torch.int8), scale


def _plain_quantise_blocks(x):
    """x [R, C] -> (float8_e4m3fn [R, C], float8_e8m0fnu [C / 512 rounded up, R, 4]): a power of two for each 128 of a row"""
    R, C = x.shape
    Cb = -(-C // BLOCK)
    blocks = torch.zeros(R, Cb * BLOCK, device=x.device)
    blocks[:, :C] = x
    blocks = blocks.view(R, Cb, BLOCK)
    top = blocks.abs().amax(dim=2)
    frac, expo = torch.frexp(top)                                         # top = frac 2^expo, frac in [0.5, 1)
    expo = torch.where(frac > 0.875, expo - 8, expo - 9).clamp(min=-127)  # 448 = 0.875 * 2^9
    expo = torch.where(top > 0, expo, torch.zeros_like(expo))
    q = torch.ldexp(blocks.double(), -expo[:, :, None]).float().to(torch.float8_e4m3fn)
    scale = torch.full((R, -(-Cb // 4) * 4), 127, dtype=torch.uint8, device=x.device)
    scale[:, :Cb] = (expo + 127).to(torch.uint8)
    scale = scale.view(R, -1, 4).transpose(0, 1).contiguous()
    return q.view(R, Cb * BLOCK)[:, :C].contiguous(), scale.view(torch.float8_e8m0fnu)


def _plain_norm(st):
    """(normalised in fp32, the sum as it is stored and normalised, 1 / root mean square)"""
    s = st["x"].float()
    if st["residual"] is not None:
        s = (s + st["residual"].float()).to(st["x"].dtype).float()
    r = torch.rsqrt(s.square().mean(dim=1, keepdim=True) + EPS)
    return s * r * st["weight"].float(), s, r


def _plain_norm_bwd(st, s, r):
    dh, w = st["dh"].float(), st["weight"].float()
    n = s * r
    gw = dh * w
    dx = r * (gw - n * (gw * n).mean(dim=1, keepdim=True))
    if st["dsum"] is not None:
        dx = dx + st["dsum"].float()
    return dx.to(st["x"].dtype), (dh * n).sum(dim=0).to(st["weight"].dtype)


def _softmax64(z, temperature):
    z = z.double() / temperature
    e = torch.exp(z - z.amax(dim=-1, keepdim=True))
    return e / e.sum(dim=-1, keepdim=True)


def _plain_verify(st):
    z, x, lens, u = st["logits"], st["drafts"].long(), st["lens"].long(), st["uniforms"].double()
    B, K1, V = z.shape
    K = K1 - 1
    greedy = st["temperature"] == 0
    t = torch.where(greedy, torch.ones_like(st["temperature"]), st["temperature"]).double()[:, None, None]
    p = _softmax64(z, t)
    index = torch.arange(V, device=DEV)
    top = torch.where(z == z.amax(dim=2, keepdim=True), index, V).amin(dim=2)            # the first of the largest
    point = (index == top[:, :, None]).double()
    p = torch.where(greedy[:, None, None], point, p)
    if st["draft_logits"] is not None:
        q = torch.where(greedy[:, None, None], (index == x[:, :, None]).double(), _softmax64(st["draft_logits"], t))
    else:
        q = (index == x[:, :, None]).double()
    at = torch.arange(K, device=DEV)[None, :]
    px, qx = p[:, :K].gather(2, x[:, :, None])[:, :, 0], q.gather(2, x[:, :, None])[:, :, 0]
    keep = (u[:, :K] * qx < px) & (at < lens[:, None])
    a = keep.long().cumprod(dim=1).sum(dim=1)                                            # accepted drafts
    b = torch.arange(B, device=DEV)
    pa = p[b, a]
    r = pa
    if K > 0:
        left = (pa - q[b, a.clamp(max=K - 1)]).clamp(min=0)
        r = torch.where(((a < lens) & (left.sum(dim=1) > 0))[:, None], left, pa)
    c = r.cumsum(dim=1)
    y = (c <= u[:, K:] * c[:, -1:]).sum(dim=1)
    slots = torch.arange(K1, device=DEV)[None, :]
    tokens = torch.where(slots == a[:, None], y[:, None], torch.nn.functional.pad(x, (0, 1)))
    logp = torch.log(p.gather(2, tokens[:, :, None])[:, :, 0])
    past = slots > a[:, None]
    return (torch.where(past, -1, tokens).to(torch.int32), a.to(torch.int32), torch.where(past, 0.0, logp).float())


# ---- one pass -----------------------------------------------------------------------------------------------------------

def run(st):
    case, kind = st["case"], st["case"]["kind"]
    if own:
        from paper_2505_24034_amd import binding as L
    if kind == "norm":
        if own:
            h, s, r = L.rms_norm(st["x"], st["weight"], EPS, residual=st["residual"])
            dx, dw = L.rms_norm_bwd(st["dh"], s, st["weight"], r, dsum=st["dsum"])
        else:
            h, s, r = _plain_norm(st)
            dx, dw = _plain_norm_bwd(st, s, r)
            h, s, r = h.to(st["x"].dtype), s.to(st["x"].dtype), r[:, 0]
        return dict(h=h, sum=s, rstd=r, dx=dx, dw=dw)
    if kind == "norm8":
        if own:
            call = L.rms_norm_rows if case["out"] == "rows" else L.rms_norm_blocks
            q, scale, s = call(st["x"], st["weight"], EPS, residual=st["residual"])
        else:
            h, s, _ = _plain_norm(st)
            q, scale = _plain_quantise_rows(h) if case["out"] == "rows" else _plain_quantise_blocks(h)
            s = s.to(st["x"].dtype)
        return dict(q=q.to(torch.bfloat16) if case["out"] == "rows" else q, scale=scale, sum=s)
    if kind == "verify":
        if own:
            tokens, accepted, logp = L.verify_drafts(st["logits"], st["drafts"], st["uniforms"], draft_logits=st["draft_logits"],
                                                     draft_lens=st["lens"], temperature=st["temperature"])
        else:
            tokens, accepted, logp = _plain_verify(st)
        return dict(tokens=tokens, accepted=accepted, logp=logp)
    if own:
        Hq, Hs = L.quantise_rows(st["H"])
        if kind == "logits":
            return dict(z=L.logits_rows(Hq, Hs, st["Wq"], st["Ws"], dtype=_dtype(case["out"])))
        logp, lse = L.token_logprobs_rows(Hq, Hs, st["Wq"], st["Ws"], st["targets"], st["mask"].reshape(-1))
        return dict(logp=logp, lse=lse)
    Hq, Hs = _plain_quantise_rows(st["H"].float())
    z = (Hq.float() @ st["Wq"].float().T).mul_(st["Ws"]).mul_(Hs[:, None])
    if kind == "logits":
        return dict(z=z.to(_dtype(case["out"])))
    valid = st["mask"].reshape(-1) != 0
    zy = z.gather(1, st["targets"].long()[:, None])[:, 0]
    top = z.amax(dim=1)
    lse = z.sub_(top[:, None]).exp_().sum(dim=1).log() + top
    zero = torch.zeros_like(lse)
    return dict(logp=torch.where(valid, zy - lse, zero), lse=torch.where(valid, lse, zero))


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------

def work(case):
    """Every input read once, every output written once; logprobs: of the mean number of valid tokens; verify: of the mean number
    of drafts, and with half of them the rows whose distribution is asked for."""
    kind = case["kind"]
    if kind in ("norm", "norm8"):
        n, N, d = case["N"] * case["d"], case["N"], case["d"]
        e, r = 2 if case["dtype"] == "bf16" else 4, int(case["residual"])
        if kind == "norm":      # x, residual, h, sum; dh, sum, dsum, dx (the sum is x where there is no residual)
            return dict(bytes=n * e * (2 + 2 * r + 3 + r) + 8 * N + 3 * e * d, flops=16 * n)
        return dict(bytes=n * e * (1 + 2 * r) + n + 4 * N * (1 if case["out"] == "rows" else -(-d // 512)) + e * d, flops=8 * n)
    if kind == "verify":
        e = 2 if case["dtype"] == "bf16" else 4
        drafts = case["K"] / 2.0 if case["ragged"] else case["K"]
        rows = case["B"] * (drafts + 1 + (drafts if case["drafts"] == "model" else 0)) * case["V"]
        return dict(bytes=rows * e + case["B"] * (case["K"] + 1) * 16, flops=4 * rows)
    d, V = case["d"], case["V"]
    head = V * d + 4 * V
    if kind == "logits":
        N = case["N"]
        return dict(bytes=head + 2 * N * d + N * V * (2 if case["out"] == "bf16" else 4), flops=2 * N * V * d)
    N = case["B"] * case["T"]
    n = case["B"] * (case["len_lo"] + case["T"]) / 2.0
    return dict(bytes=head + 2 * n * d + 13 * N, flops=2 * n * V * d)


# ---- the definition in 64 bits --------------------------------------------------------------------------------------------

def _exact_norm(case, st):
    s = st["x"].double()
    if st["residual"] is not None:
        s = (st["x"].double() + st["residual"].double()).to(st["x"].dtype).double()
    r = (s.pow(2).sum(dim=1) / case["d"] + EPS).pow(-0.5)
    n = s * r.unsqueeze(1)
    w = st["weight"].double()
    h = n * w
    if case["kind"] == "norm":
        dh = st["dh"].double()
        proj = torch.einsum("ij,ij->i", dh * w, n) / case["d"]
        dx = (dh * w - n * proj.unsqueeze(1)) * r.unsqueeze(1)
        if st["dsum"] is not None:
            dx += st["dsum"].double()
        return dict(h=h, sum=s, rstd=r, dx=dx, dw=torch.einsum("ij,ij->j", dh, n))
    if case["out"] == "rows":
        scale = h.abs().max(dim=1).values / 127
        return dict(q=torch.round(h / scale.unsqueeze(1)), scale=scale, sum=s)
    R, C = h.shape
    Cb = (C + BLOCK - 1) // BLOCK
    table = torch.ones(R, (Cb + 3) // 4 * 4, dtype=torch.float64, device=h.device)
    for b in range(Cb):
        cols = slice(b * BLOCK, min(C, (b + 1) * BLOCK))
        e = torch.ceil(torch.log2(h[:, cols].abs().max(dim=1).values / E4M3_MAX))
        e = torch.where(torch.isfinite(e), e, torch.zeros_like(e))
        table[:, b] = torch.exp2(e)
        h[:, cols] /= table[:, b, None]
    return dict(q=h, scale=table.unflatten(1, (-1, 4)).permute(1, 0, 2).contiguous(), sum=s)


def _exact_verify(case, st):
    """One sequence after the other, as the method is stated."""
    B, K, V = case["B"], case["K"], case["V"]
    tokens = torch.full((B, K + 1), -1, dtype=torch.int32)
    accepted = torch.zeros(B, dtype=torch.int32)
    logp = torch.zeros(B, K + 1, dtype=torch.float64)
    drafts, u, lens, temp = (st[k].cpu() for k in ("drafts", "uniforms", "lens", "temperature"))

    def dist(row, T):
        if T == 0:
            first = int((row == row.max()).nonzero()[0])
            e = torch.zeros(V, dtype=torch.float64, device=row.device)
            e[first] = 1
            return e
        return torch.softmax(row.double() / T, dim=0)

    for b in range(B):
        T, n = float(temp[b]), int(lens[b])
        for i in range(n + 1):
            p = dist(st["logits"][b, i], T)
            if i < n:
                x = int(drafts[b, i])
                if st["draft_logits"] is not None and T > 0:
                    q = dist(st["draft_logits"][b, i], T)
                else:
                    q = torch.zeros_like(p)
                    q[x] = 1
                if float(u[b, i]) * float(q[x]) < float(p[x]):
                    tokens[b, i] = x
                    logp[b, i] = math.log(float(p[x]))
                    continue
                r = torch.relu(p - q)
                r = r if float(r.sum()) > 0 else p
            else:
                r = p
            c = torch.cumsum(r, dim=0)
            y = int(torch.searchsorted(c, c[-1:] * float(u[b, K]), right=True))
            tokens[b, i], accepted[b], logp[b, i] = y, i, math.log(float(p[y]))
            break
    return dict(tokens=tokens.to(DEV), accepted=accepted.to(DEV), logp=logp.to(DEV))


def exact(case, seed):
    with torch.no_grad():
        st = prepare(case, seed)
        if case["kind"] in ("norm", "norm8"):
            return _exact_norm(case, st)
        if case["kind"] == "verify":
            return _exact_verify(case, st)
        H = st["H"].float()
        s = (H.abs().max(dim=1).values.double() / 127).float().unsqueeze(1)
        H = torch.round(H / s).double() * s.double()
        W = st["Wq"].double() * st["Ws"].double().unsqueeze(1)
        if case["kind"] == "logits":
            return dict(z=torch.cat([h @ W.T for h in H.split(1024)]))
        N = H.shape[0]
        logp = torch.zeros(N, dtype=torch.float64, device=DEV)
        lse = torch.zeros(N, dtype=torch.float64, device=DEV)
        for rows in st["mask"].reshape(-1).nonzero()[:, 0].split(1024):
            z = H[rows] @ W.T
            lse[rows] = torch.logsumexp(z, dim=1)
            logp[rows] = z[torch.arange(rows.numel(), device=DEV), st["targets"][rows].long()] - lse[rows]
        return dict(logp=logp, lse=lse)
