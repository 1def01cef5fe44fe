"""Measured operators: the update that follows the head's gradients, and the head in 8 bits that a generator works with.

A case is a dict of plain values; `kind` says which pass it makes:

  adamw      grad_norm over a model's gradients and adamw_step with the clip scale, on states in 32 or 8 bits
  quantise   quantise_blocks of a matrix: activations in rows of 128, weights in blocks of 128 x 128
  logits     hidden states quantised and multiplied with an 8-bit head: what a decoding step or a prompt's scoring does
  logprobs   the log-probabilities of given tokens under that head (the generator's mu), without logits in memory

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
LR, BETA1, BETA2, EPS, DECAY = 1e-4, 0.9, 0.999, 1e-8, 0.01
TINY_SCALE = 2.0 ** -100          # a block of states below this is zeros


def listed():
    return [
        # a unit-test sized fp32 model: nineteen tensors, launch latency counts
        dict(name="adamw32_tiny", kind="adamw", bits=32, V=1024, d=256, f=680, kv=64, layers=2, param="f32", grad="f32", clip=True),
        # a ~170 M model: 109 tensors of very different sizes, bf16 weights with fp32 copies
        dict(name="adamw32_model", kind="adamw", bits=32, V=33001, d=1032, f=2752, kv=258, layers=12, param="bf16", grad="bf16",
             clip=True),
        # the 8B head alone, its gradient accumulated in fp32
        dict(name="adamw32_8b_head", kind="adamw", bits=32, V=FULL_V, d=4096, f=0, kv=0, layers=0, param="bf16", grad="f32",
             clip=True),
        # a small model with no size a multiple of a block, states in 8 bits
        dict(name="adamw8_small_odd", kind="adamw", bits=8, V=5003, d=523, f=1391, kv=131, layers=3, param="bf16", grad="bf16",
             clip=True),
        # the 8B head with 8-bit states: memory-bound trainer, no clip
        dict(name="adamw8_8b_head", kind="adamw", bits=8, V=FULL_V, d=4096, f=0, kv=0, layers=0, param="bf16", grad="bf16",
             clip=False),
        # the 8B head goes to the generator after an update
        dict(name="quantise_8b_head", kind="quantise", rows=FULL_V, d=4096, dtype="bf16", block_rows=128),
        # hidden states of one micro-batch, rows that end inside a block
        dict(name="quantise_hidden_odd", kind="quantise", rows=1901, d=1040, dtype="bf16", block_rows=1),
        # one decoding step of one sequence at the 8B head: the weights' bytes are the time
        dict(name="logits_8b_one_token", kind="logits", N=1, d=4096, V=FULL_V, out="f32"),
        # a decoding step of 48 sequences on one of eight ranks of the 70B head
        dict(name="logits_70b_rank_48", kind="logits", N=48, d=8192, V=16032, out="f32"),
        # a prompt's logits under a ~1B-class head
        dict(name="logits_1b_prompt", kind="logits", N=1900, d=2048, V=33001, out="bf16"),
        # a debugging run: no size a multiple of a tile
        dict(name="logprobs_small_odd", kind="logprobs", B=3, T=347, len_lo=40, d=528, V=5003),
        # mu of a trainer batch at the 8B shape
        dict(name="logprobs_8b", kind="logprobs", B=8, T=2048, len_lo=256, d=4096, V=FULL_V),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["adamw", "adamw", "quantise", "logits", "logits", "logprobs"])
    if kind == "adamw":
        while True:
            d = _log_int(rng, 64, 4096)
            layers = rng.choice([0, 1, 2, 4, 12, 24])
            case = dict(kind=kind, bits=rng.choice([8, 32]), V=_log_int(rng, 500, FULL_V), d=d, f=_log_int(rng, d, 4 * d),
                        kv=max(1, d // rng.choice([1, 4, 8])), layers=layers, param=rng.choice(["bf16", "f32"]),
                        grad=rng.choice(["bf16", "f32"]), clip=rng.random() < 0.7)
            if sum(_sizes(case)) <= FULL_V * 4096 * 3 // 4:
                return case
    d = 16 * _log_int(rng, 8, 512)
    if kind == "quantise":
        return dict(kind=kind, rows=_log_int(rng, 1, min(FULL_V, FULL_V * 4096 // d)), d=d, dtype=rng.choice(["bf16", "f32"]),
                    block_rows=rng.choice([1, 128]))
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
    g.manual_seed(1000003 * seed + 11)
    return g


def _rand(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _dtype(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _sizes(case):
    """entries of each tensor: the head, then per layer q, k, v, o, gate, up, down and two norms"""
    d, f, kv = case["d"], case["f"], case["kv"]
    return [case["V"] * d] + case["layers"] * [d * d, kv * d, kv * d, d * d, f * d, f * d, d * f, d, d]


def _prepare_adamw(case, seed):
    g = _gen(seed)
    sizes = _sizes(case)
    starts = [0]
    for n in sizes:
        starts.append(starts[-1] + (n + BLOCK - 1) // BLOCK * BLOCK)      # tensors start on whole blocks of one buffer
    total = starts[-1]
    param, grad = _dtype(case["param"]), _dtype(case["grad"])
    master = torch.zeros(total, device=DEV)
    G = torch.zeros(total, dtype=grad, device=DEV)
    m = torch.zeros(total, device=DEV)
    r = torch.zeros(total, device=DEV)                                    # square root of the second moment
    for i, n in enumerate(sizes):
        at = slice(starts[i], starts[i] + n)
        size = 1e-3 * 10.0 ** ((i % 5) / 2.0 - 1.0)                       # gradients of a model's tensors differ in size
        master[at] = _rand(g, n).mul_(case["d"] ** -0.5)
        spread = torch.rand(n, generator=g, device=DEV).add_(0.25)        # ... and those of a tensor's entries
        G[at] = (_rand(g, n) * spread * size).to(grad)
        m[at] = _rand(g, n).mul_(spread).mul_(0.25 * size)
        r[at] = spread.mul_(size)
        del spread
    st = dict(case=case, step=200, sizes=sizes, starts=starts, G=G, starts_dev=torch.tensor(starts[:-1], device=DEV))
    if param == torch.float32:
        st["p"], st["master"] = master, None
    else:
        st["p"], st["master"] = master.to(param), master
    if case["bits"] == 32:
        st.update(m=m, v=r.square_(), m_scale=None, v_scale=None)
    else:
        for name, x in (("m", m), ("v", r)):
            s = x.view(-1, BLOCK).abs().amax(dim=1) / E4M3_MAX
            st[name] = (x.view(-1, BLOCK) / s.clamp(min=1e-30)[:, None]).to(torch.float8_e4m3fn).view(-1)
            st[name + "_scale"] = s
    views = {}
    for name in ("p", "G", "m", "v", "master"):
        views[name] = None if st[name] is None else [st[name][a:a + n] for a, n in zip(starts, sizes)]
    for name in ("m_scale", "v_scale"):
        views[name] = None if st[name] is None else [st[name][a // BLOCK:(a + n + BLOCK - 1) // BLOCK] for a, n in zip(starts, sizes)]
    st["views"] = views
    return st


def _plain_quantise(x, block_rows):
    """x [R, C] -> (q float8_e4m3fn [R, C], scale float8_e8m0fnu [C / 512 rounded up, R or ceil(R / 128), 4])"""
    R, C = x.shape
    Rb, Cb = -(-R // block_rows), -(-C // BLOCK)
    blocks = torch.zeros(Rb * block_rows, Cb * BLOCK, device=x.device)
    blocks[:R, :C] = x
    blocks = blocks.view(Rb, block_rows, Cb, BLOCK)
    finite = blocks.isfinite()
    top = torch.where(finite, blocks.abs(), torch.zeros_like(blocks)).amax(dim=(1, 3))
    frac, expo = torch.frexp(top)                                         # top = frac 2^expo, frac in [0.5, 1)
    expo = torch.where(frac > 0.875, expo - 8, expo - 9).clamp(min=-127)  # 448 = 0.875 * 2^9
    expo = torch.where(top > 0, expo, torch.zeros_like(expo))
    q = torch.ldexp(blocks.double(), -expo[:, None, :, None])             # exact: powers of two
    q = torch.where(finite, q, torch.full_like(q, math.nan)).float().to(torch.float8_e4m3fn)
    scale = torch.full((Rb, -(-Cb // 4) * 4), 127, dtype=torch.uint8, device=x.device)
    scale[:, :Cb] = (expo + 127).to(torch.uint8)
    scale = scale.view(Rb, -1, 4).transpose(0, 1).contiguous()
    return q.view(Rb * block_rows, Cb * BLOCK)[:R, :C].contiguous(), scale.view(torch.float8_e8m0fnu)


def _plain_dequantise(q, scale, block_rows):
    R, C = q.shape
    s = scale.float().transpose(0, 1).flatten(1)[:, :-(-C // BLOCK)].repeat_interleave(BLOCK, dim=1)[:, :C]
    return q.float() * s.repeat_interleave(block_rows, dim=0)[:R]


def _mask(g, B, T, len_lo):
    lens = len_lo + torch.floor(torch.rand(B, generator=g, device=DEV) * (T - len_lo + 1)).long().clamp_(max=T - len_lo)
    return (torch.arange(T, device=DEV)[None, :] < lens[:, None]).to(torch.uint8).contiguous()


def prepare(case, seed):
    if case["kind"] == "adamw":
        return _prepare_adamw(case, seed)
    g = _gen(seed)
    d = case["d"]
    if case["kind"] == "quantise":
        x = _rand(g, case["rows"], d)
        x *= torch.exp(0.5 * _rand(g, 1, d))                              # channels of different size, some of them outliers
        return dict(case=case, x=(x * d ** -0.5).to(_dtype(case["dtype"])).contiguous())
    N = case["N"] if case["kind"] == "logits" else case["B"] * case["T"]
    H = _rand(g, N, d).to(torch.bfloat16)                                 # after the final norm
    Wq, Ws = _plain_quantise((_rand(g, case["V"], d) * d ** -0.5).to(torch.bfloat16), BLOCK)
    st = dict(case=case, H=H, Wq=Wq, Ws=Ws)
    if case["kind"] == "logprobs":
        st["mask"] = _mask(g, case["B"], case["T"], case["len_lo"])
        st["targets"] = torch.randint(0, case["V"], (N,), generator=g, device=DEV).to(torch.int32)
    return st


# ---- one pass -----------------------------------------------------------------------------------------------------------

def _noise(st, step):
    """16 random bits for each entry of the flat buffer, hashed out of the step, the tensor's place in the list and the entry's
    place in the tensor; two neighbouring entries share a 32-bit hash"""
    low = 0xFFFFFFFF
    i = torch.arange(st["p"].numel(), device=DEV)
    t = torch.bucketize(i, st["starts_dev"], right=True) - 1
    i -= st["starts_dev"][t]
    x = ((i >> 1) + step * 0x9E3779B9 + t * 0xB504F333) & low
    x = ((x ^ (x >> 16)) * 0xDDB3D743) & low
    x = ((x ^ (x >> 15)) * 0x8F1BBCDD) & low
    x = x ^ (x >> 16)
    return torch.where((i & 1) == 1, x >> 16, x & 0xFFFF)


def _plain_hold(x, noise):
    """x [blocks, 128] as (float8_e4m3fn, scale): to nearest, or stochastically with `noise`; nothing positive becomes zero then"""
    top = x.abs().amax(dim=1)
    scale = torch.where(top < TINY_SCALE, torch.zeros_like(top), top / E4M3_MAX)
    y = torch.where(scale[:, None] > 0, x / scale[:, None], torch.zeros_like(x))
    if noise is not None:
        lift = torch.where(y < 2.0 ** -6, 2.0 ** -6, 0.0)                 # below the normal numbers the steps are those above
        z = (y + lift).view(torch.int32)
        z = ((z + (noise.view_as(z) << 4).to(torch.int32)) & -(1 << 20)).view(torch.float32) - lift
        y = torch.where(y > 0, z.clamp(2.0 ** -9, E4M3_MAX), torch.zeros_like(z))
    return y.to(torch.float8_e4m3fn), scale


def _plain_adamw(st, step):
    case = st["case"]
    g = st["G"].float()
    norm = g.double().square().sum().sqrt()
    if case["clip"]:
        g = g * torch.where(norm > 1.0, 1.0 / norm, torch.ones_like(norm)).float()
    p = (st["p"] if st["master"] is None else st["master"])
    if case["bits"] == 32:
        m, v = st["m"], st["v"]
        m.mul_(BETA1).add_(g * (1 - BETA1))
        v.mul_(BETA2).add_(g.square() * (1 - BETA2))
        r = v.sqrt()
    else:
        m = (st["m"].float().view(-1, BLOCK) * st["m_scale"][:, None]).view(-1) * BETA1 + g * (1 - BETA1)
        r = (st["v"].float().view(-1, BLOCK) * st["v_scale"][:, None]).view(-1)
        r = (r.square() * BETA2 + g.square() * (1 - BETA2)).sqrt()
        for name, x, noise in (("m", m, None), ("v", r, _noise(st, step))):
            q, s = _plain_hold(x.view(-1, BLOCK), noise)
            st[name].copy_(q.view(-1))
            st[name + "_scale"].copy_(s)
    c1, c2 = 1 - BETA1 ** step, 1 - BETA2 ** step
    p.sub_((p * DECAY + (m / c1) / (r / math.sqrt(c2) + EPS)) * LR)
    if st["master"] is not None:
        st["p"].copy_(p)
    return norm.float().view(1)


def _adamw_outputs(st, norm):
    out = dict(p=st["p"], m=st["m"], v=st["v"])
    if st["master"] is not None:
        out["master"] = st["master"]
    if st["m_scale"] is not None:
        out.update(m_scale=st["m_scale"], v_scale=st["v_scale"])
    if norm is not None:
        out["norm"] = norm
    return out


def run(st):
    case = st["case"]
    if own:
        from paper_2505_24034_amd import binding as L
    if case["kind"] == "adamw":
        st["step"] += 1
        if own:
            w = st["views"]
            norm, scale = L.grad_norm(w["G"], 1.0) if case["clip"] else (None, None)
            L.adamw_step(w["p"], w["G"], w["m"], w["v"], LR, st["step"], betas=(BETA1, BETA2), eps=EPS, weight_decay=DECAY,
                         masters=w["master"], exp_avg_scales=w["m_scale"], exp_avg_sq_scales=w["v_scale"], grad_scale=scale)
        else:
            norm = _plain_adamw(st, st["step"])
        return _adamw_outputs(st, norm if case["clip"] else None)
    if case["kind"] == "quantise":
        q, s = L.quantise_blocks(st["x"], case["block_rows"]) if own else _plain_quantise(st["x"].float(), case["block_rows"])
        return dict(q=q, scale=s)
    if own:
        Hq, Hs = L.quantise_blocks(st["H"], 1)
        if case["kind"] == "logits":
            return dict(z=L.logits_blocks(Hq, Hs, st["Wq"], st["Ws"], dtype=_dtype(case["out"])))
        logp, lse = L.token_logprobs_blocks(Hq, Hs, st["Wq"], st["Ws"], st["targets"], st["mask"].reshape(-1))
        return dict(logp=logp, lse=lse)
    Hq, Hs = _plain_quantise(st["H"].float(), 1)
    z = _plain_dequantise(Hq, Hs, 1) @ _plain_dequantise(st["Wq"], st["Ws"], BLOCK).T
    if case["kind"] == "logits":
        return dict(z=z.to(_dtype(case["out"])))
    valid = st["mask"].reshape(-1) != 0
    zy = z.gather(1, st["targets"].long()[:, None])[:, 0]
    top = z.amax(dim=1)
    lse = z.sub_(top[:, None]).exp_().sum(dim=1).log() + top
    zero = torch.zeros_like(lse)
    return dict(logp=torch.where(valid, zy - lse, zero), lse=torch.where(valid, lse, zero))


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------

def _scale_columns(d):
    return -(-d // (4 * BLOCK)) * 4


def work(case):
    """Every input read once, every output written once; logprobs: of the mean number of valid tokens."""
    kind, d = case["kind"], case["d"]
    if kind == "adamw":
        n = sum(_sizes(case))
        p = 2 + 4 + 4 if case["param"] == "bf16" else 4 + 4
        state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
        return dict(bytes=n * (p + state + (2 if case["grad"] == "bf16" else 4)), flops=(18 if case["clip"] else 16) * n)
    if kind == "quantise":
        n = case["rows"] * d
        return dict(bytes=n * (3 if case["dtype"] == "bf16" else 5) + -(-case["rows"] // case["block_rows"]) * _scale_columns(d), flops=2 * n)
    V = case["V"]
    head = V * d + -(-V // BLOCK) * _scale_columns(d)
    if kind == "logits":
        N = case["N"]
        return dict(bytes=head + 2 * N * d + N * V * (2 if case["out"] == "bf16" else 4), flops=2 * N * V * d)
    N = case["B"] * case["T"]
    n = case["B"] * (case["len_lo"] + case["T"]) / 2.0
    return dict(bytes=head + 2 * n * d + 13 * N, flops=2 * n * V * d)


# ---- the definition in 64 bits --------------------------------------------------------------------------------------------

def _exact_block_scale(x, block_rows):
    """exponent of every entry's block, [R, C], and the table of scales"""
    R, C = x.shape
    Rb, Cb = (R + block_rows - 1) // block_rows, (C + BLOCK - 1) // BLOCK
    a = torch.nn.functional.pad(x.abs(), (0, Cb * BLOCK - C, 0, Rb * block_rows - R))
    top = a.unflatten(1, (Cb, BLOCK)).amax(dim=2).unflatten(0, (Rb, block_rows)).amax(dim=1).double()
    del a
    e = torch.ceil(torch.log2(top / E4M3_MAX))
    e = torch.where(top / E4M3_MAX * torch.exp2(-e) > 1, e + 1, e)        # the logarithm is rounded: settle the borders
    e = torch.where(top / E4M3_MAX * torch.exp2(-e) <= 0.5, e - 1, e)
    e = torch.where(top > 0, e.clamp(min=-127), torch.zeros_like(e))
    table = torch.ones(Rb, (Cb + 3) // 4 * 4, dtype=torch.float64, device=x.device)
    table[:, :Cb] = torch.exp2(e)
    full = table[:, :Cb].repeat_interleave(BLOCK, dim=1)[:, :C].repeat_interleave(block_rows, dim=0)[:R]
    return full, table.unflatten(1, (-1, 4)).permute(1, 0, 2).contiguous()


def _exact_adamw(case, seed):
    st = _prepare_adamw(case, seed)
    t = st["step"] + 1
    G = st["G"].double()
    norm = torch.linalg.vector_norm(G)
    if case["clip"] and float(norm) > 1.0:
        G /= norm
    lens = torch.tensor(st["starts"], device=DEV).diff() // BLOCK

    def held(name):
        if case["bits"] == 32:
            return st[name].double()
        x = st[name].double().unflatten(0, (-1, BLOCK)) * st[name + "_scale"].double().unsqueeze(1)
        return x.flatten()

    m = torch.lerp(G, held("m"), BETA1)
    v = held("v") if case["bits"] == 32 else held("v").square()
    v = torch.lerp(G.square(), v, BETA2)
    del G
    p = (st["p"] if st["master"] is None else st["master"]).double()
    update = (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)).sqrt() + EPS)
    p -= LR * (DECAY * p + update)
    del update
    out = dict(p=p)
    if st["master"] is not None:
        out["master"] = p
    if case["bits"] == 32:
        out.update(m=m, v=v)
    else:                                                                  # before they are rounded to 8 bits
        for name, x in (("m", m), ("v", v.sqrt())):
            s = x.unflatten(0, (int(lens.sum()), BLOCK)).abs().amax(dim=1) / E4M3_MAX
            out[name + "_scale"] = s
            out[name] = x / s.clamp(min=1e-300).repeat_interleave(BLOCK)
    if case["clip"]:
        out["norm"] = norm.reshape(1)
    return out


def exact(case, seed):
    with torch.no_grad():
        if case["kind"] == "adamw":
            return _exact_adamw(case, seed)
        st = prepare(case, seed)
        if case["kind"] == "quantise":
            s, table = _exact_block_scale(st["x"], case["block_rows"])
            return dict(q=st["x"].double() / s, scale=table)
        d = case["d"]
        s, _ = _exact_block_scale(st["H"], 1)
        H = (st["H"].double() / s).to(torch.float8_e4m3fn).double() * s    # the quotient is exact in bf16's bits
        table = st["Ws"].double().permute(1, 0, 2).flatten(1)
        W = st["Wq"].double()
        for b in range((d + BLOCK - 1) // BLOCK):
            W[:, b * BLOCK:(b + 1) * BLOCK] *= table[:, b].repeat_interleave(BLOCK)[:W.shape[0], None]
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
