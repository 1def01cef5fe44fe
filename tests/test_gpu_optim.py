"""llamarl_grad_norm, llamarl_adamw_step and the optimiser over them, against the formulas in 64 bits.

u = 2^-24 is half a step of fp32.  m is one fma of a rounded product with rounded factors: within 5 u of |b1 m| + |(1 - b1) g|; v, whose terms
are positive, within 7 u of itself.  The update m / c1 / (sqrt(v / c2) + eps) takes a root and a reciprocal of 1 ulp (2 u) each and five
more roundings: within 24 u of the update formed with |b1 m| + |(1 - b1) g|.  What a parameter adds is its own last rounding:
u (fp32) or 2^-8 (bf16)."""
import numpy as np
import pytest
import torch

from operator_util import BLOCK, E4M3_MAX, adamw, blocks_of, e4m3_nearest, e4m3_values, f64, rounding_bits

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SIZES = [1, 7, 8, 9, 0, 127, 128, 129, 1023, 2048, 2049, 4097, 33333]


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _make(n, g, param=torch.float32, grad=torch.float32, bits=32, master=False, shift=0, fresh=False):
    """one tensor's arrays; shift: entries by which every array starts behind a 16-byte boundary"""
    def at(x):
        y = torch.empty(n + shift, dtype=x.dtype, device="cuda")[shift:]
        return y.copy_(x)

    def rand(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    t = dict(n=n, bits=bits, ms=None, vs=None, master=None)
    w = 0.02 * rand(n)
    t["p"] = at(w.to(param))
    if master:
        t["master"] = at(w)
    t["g"] = at((1e-3 * rand(n) * 10.0 ** (2.0 * torch.rand(n, generator=g, device="cuda") - 1.0)).to(grad))
    m, r = 3e-4 * rand(n), 1e-3 * (0.3 + torch.rand(n, generator=g, device="cuda"))
    if fresh:
        m, r = torch.zeros_like(m), torch.zeros_like(r)
    if bits == 32:
        t["m"], t["v"] = at(m), at(r * r)
    else:
        for name, x in (("m", m), ("v", r)):
            rows = torch.zeros(-(-n // BLOCK) * BLOCK, device="cuda")
            rows[:n] = x
            s = rows.view(-1, BLOCK).abs().amax(1) / E4M3_MAX
            t[name + "s"] = s
            q = (rows.view(-1, BLOCK) / s.clamp(min=1e-30)[:, None]).view(-1)[:n].to(torch.float8_e4m3fn)
            t[name] = torch.empty(n + shift, dtype=torch.uint8, device="cuda")[shift:].view(torch.float8_e4m3fn)
            t[name].view(torch.uint8).copy_(q.view(torch.uint8))
    return t


def _lists(ts):
    return {k: [t[k] for t in ts] for k in ("p", "g", "m", "v", "master", "ms", "vs")}


def _run(lib, ts, lr, step, stream=None, **kw):
    x = _lists(ts)
    lib.adamw_step(x["p"], x["g"], x["m"], x["v"], lr, step, masters=x["master"], exp_avg_scales=x["ms"], exp_avg_sq_scales=x["vs"],
                   stream=stream, **kw)


def _clone(ts):
    return [{k: v.clone() if torch.is_tensor(v) else v for k, v in t.items()} for t in ts]


def _bits(ts):
    out = []
    for t in ts:
        out += [v.view(torch.uint8) if v.dtype == torch.float8_e4m3fn else v for k, v in sorted(t.items()) if torch.is_tensor(v)]
    return out


def _same(a, b):
    return all(torch.equal(x, y) for x, y in zip(_bits(a), _bits(b)))


def _held(t, name):
    if t["bits"] == 32:
        return f64(t[name])
    s = np.repeat(f64(t[name + "s"]), BLOCK)[:t["n"]]
    x = e4m3_values(t[name]) * s
    return x * x if name == "v" else x


def _check(before, after, place, lr, t, betas, eps, wd, scale):
    b1, b2 = betas
    n = before["n"]
    p0 = f64(before["p"] if before["master"] is None else before["master"])
    m0, v0, g = _held(before, "m"), _held(before, "v"), f64(before["g"])
    p, m, v = adamw(p0, g, m0, v0, lr, t, b1, b2, eps, wd, scale)
    top = b1 * np.abs(m0) + (1 - b1) * np.abs(g * scale)
    move = top / (1 - b1 ** t) / (np.sqrt(v / (1 - b2 ** t)) + eps)
    tol = U * np.abs(p) + lr * (4 * U * wd * np.abs(p0) + 24 * U * move) + 1e-44
    moved = after["p"] if after["master"] is None else after["master"]
    if moved.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * np.abs(p)
    assert (np.abs(f64(moved) - p) <= tol).all(), "parameter"
    if after["master"] is not None:
        assert torch.equal(after["p"], after["master"].to(torch.bfloat16))
    if before["bits"] == 32:
        assert (np.abs(f64(after["m"]) - m) <= 5 * U * top + 1e-44).all(), "first moment"
        assert (np.abs(f64(after["v"]) - v) <= 7 * U * v + 1e-44).all(), "second moment"
        return
    for name, x in (("m", m), ("v", np.sqrt(v))):
        rows = blocks_of(x)
        s = np.abs(rows).max(axis=1) / E4M3_MAX
        got = f64(after[name + "s"])
        assert (np.abs(got - s) <= 10 * U * s).all(), "factors"
        assert (got[s < 2.0 ** -101 / E4M3_MAX] == 0).all()
        y = np.divide(rows, s[:, None], out=np.zeros_like(rows), where=s[:, None] > 0).reshape(-1)[:n]
        q = e4m3_values(after[name])
        assert np.isfinite(q).all()
        a = np.abs(y)
        if name == "m":
            # Half a step, and what 12 u of y can do at a border.  How many entries fall on the other side is not counted: with b1 = 0
            # m is the bf16 gradient times the scale, and 448 m / top meets exact ties (m / top = 13 / 448), which the factor's own
            # rounding turns either way.
            assert (np.abs(q - y) <= np.maximum(2.0 ** -4 * a, 2.0 ** -10) * (1 + 2.0 ** -15) + 12 * U * E4M3_MAX).all()
        else:
            assert ((q > 0) == (y > 0)).all(), "a second moment vanished, or came out of nothing"
            bits = rounding_bits(n, t, place) / 65536.0
            expo = np.floor(np.log2(np.maximum(a, 2.0 ** -6)))
            ulp = 2.0 ** (expo - 3)
            at = a / ulp + bits
            want = np.where(y > 0, np.clip(np.floor(at) * ulp, 2.0 ** -9, E4M3_MAX), 0.0)
            assert (np.abs(q - want) <= ulp * (1 + 1e-9)).all()
            # y is within 16 u of itself, a / ulp at most 16: only an entry that near to a whole number of steps may fall on the other side
            assert ((q == want) | (np.abs(at - np.round(at)) <= 256 * U)).all()


@pytest.mark.parametrize("param,grad,master", [(torch.float32, torch.float32, False), (torch.float32, torch.bfloat16, False),
                                               (torch.bfloat16, torch.bfloat16, True), (torch.bfloat16, torch.float32, False)])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [0, 1])
def test_step_matches_the_formula(lib, param, grad, master, bits, shift):
    g = _gen(bits + shift)
    ts = [_make(n, g, param, grad, bits, master, shift) for n in SIZES]
    for lr, t, betas, eps, wd, scale in ((1e-3, 1, (0.9, 0.999), 1e-8, 0.01, None), (3e-4, 1000, (0.9, 0.95), 1e-6, 0.1, 0.37),
                                         (1e-2, 7, (0.0, 0.0), 1e-3, 0.0, 2.5)):
        before = _clone(ts)
        s = None if scale is None else torch.tensor([scale], device="cuda")
        _run(lib, ts, lr, t, betas=betas, eps=eps, weight_decay=wd, grad_scale=s)
        for i, (b, a) in enumerate(zip(before, ts)):
            assert torch.equal(a["g"], b["g"])
            _check(b, a, i, lr, t, betas, eps, wd, 1.0 if scale is None else float(np.float32(scale)))


def test_lists_longer_than_a_launch_and_of_mixed_types(lib):
    g = _gen(5)
    kinds = [dict(bits=8, param=torch.bfloat16, master=True), dict(bits=32), dict(bits=8, grad=torch.bfloat16),
             dict(bits=32, param=torch.bfloat16, shift=1), dict(bits=8, shift=3)]
    ts = [_make(SIZES[i % len(SIZES)] + i, g, **kinds[i % len(kinds)]) for i in range(131)]
    before = _clone(ts)
    again = _clone(ts)
    _run(lib, ts, 1e-3, 12)
    for i, (b, a) in enumerate(zip(before, ts)):
        _check(b, a, i, 1e-3, 12, (0.9, 0.999), 1e-8, 0.01, 1.0)
    _run(lib, again, 1e-3, 12)
    assert _same(ts, again)                                                # the same call gives the same bits


def test_fresh_states_zero_gradients_and_extreme_values(lib):
    for bits in (32, 8):
        g = _gen(6)
        t = _make(1000, g, bits=bits, fresh=True)
        t["g"][::2] = 0.0
        t["g"][128:256] = 0.0                                              # a block that stays zero
        t["g"][256:384] *= 1e-36                                           # below STATE_TINY, and squares that vanish
        t["g"][384:512] *= 1e18
        before = _clone([t])[0]
        _run(lib, [t], 1e-3, 1)
        moved = (t["p"] != before["p"] * (1 - 1e-5))
        assert torch.isfinite(t["p"]).all() and moved[1::2][:60].any()
        if bits == 8:
            assert (t["ms"][1:2] == 0).all() and (t["vs"][1:2] == 0).all()
            assert (t["m"].view(torch.uint8)[128:256] & 127 == 0).all() and (t["v"].view(torch.uint8)[128:256] == 0).all()
        keep = np.r_[0:256, 512:1000]
        for name in ("p", "m", "v"):
            for x in (before, t):
                x[name] = x[name].view(torch.uint8)[keep].view(x[name].dtype) if x[name].dtype == torch.float8_e4m3fn else x[name][keep]
        for x in (before, t):
            x["g"], x["n"] = x["g"][keep], len(keep)
            if bits == 8:
                rows = [0, 1, 4, 5, 6, 7]
                x["ms"], x["vs"] = x["ms"][rows], x["vs"][rows]
        if bits == 32:
            _check(before, t, 0, 1e-3, 1, (0.9, 0.999), 1e-8, 0.01, 1.0)


def test_states_in_8_bits_are_the_formulas_in_fp32_to_the_bit(lib):
    """operation by operation in IEEE fp32: codes and factors equal, so that whoever repeats a step elsewhere goes on alike"""
    f = np.float32
    t = _make(1 << 20, _gen(20), bits=8)
    t["g"][::3] *= 100.0
    for step in (1, 2, 3):
        g = (f64(t["g"]).astype(f) * f(0.7)).reshape(-1, BLOCK)
        m = e4m3_values(t["m"]).astype(f).reshape(-1, BLOCK) * f64(t["ms"]).astype(f)[:, None]
        r = e4m3_values(t["v"]).astype(f).reshape(-1, BLOCK) * f64(t["vs"]).astype(f)[:, None]
        m = m * f(0.9) + g * f(1 - 0.9)
        r = np.sqrt(r * r * f(0.999) + g * g * f(1 - 0.999))
        _run(lib, [t], 1e-3, step, grad_scale=torch.tensor([0.7], device="cuda"))
        sm, sr = np.abs(m).max(axis=1) * f(1 / 448), r.max(axis=1) * f(1 / 448)
        assert m.dtype == r.dtype == sm.dtype == f
        assert np.array_equal(f64(t["ms"]).astype(f), sm) and np.array_equal(f64(t["vs"]).astype(f), sr)
        y = m / sm[:, None]
        assert np.array_equal(e4m3_values(t["m"]).reshape(-1, BLOCK), e4m3_nearest(np.clip(y.astype(np.float64), -448, 448)))
        y = r / sr[:, None]
        lift = np.where(y < f(2.0 ** -6), f(2.0 ** -6), f(0))
        z = (((y + lift).view(np.int32) + (rounding_bits(y.size, step, 0).astype(np.int32) << 4).reshape(y.shape)) & ~0xFFFFF).view(f) - lift
        assert np.array_equal(e4m3_values(t["v"]).reshape(-1, BLOCK), np.where(y > 0, np.clip(z, 2.0 ** -9, 448.0), 0.0))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_no_step_with_a_scale_that_is_not_finite(lib, bad):
    g = _gen(7)
    ts = [_make(n, g, torch.bfloat16, torch.bfloat16, bits, True) for n in (5, 4000) for bits in (8, 32)]
    before = _clone(ts)
    _run(lib, ts, 1e-3, 3, grad_scale=torch.tensor([bad], device="cuda"))
    assert _same(before, ts)


def test_gradient_that_is_not_finite_stays_where_it_is(lib):
    """without a scale: the entry itself in fp32, its block of 128 at most in 8 bits"""
    for bits in (32, 8):
        t = _make(1024, _gen(8), bits=bits)
        t["g"][300] = float("nan")
        t["g"][700] = float("inf")
        _run(lib, [t], 1e-3, 3)
        ok = torch.isfinite(t["p"])
        assert not ok[300] and not ok[700]
        _run(lib, [t], 1e-3, 4)
        ok = torch.isfinite(t["p"])
        bad = ~ok
        bad[256:384] = bad[640:768] = False
        assert not bad.any() and (bits == 8 or int((~ok).sum()) == 2)


def test_step_and_rate_on_the_device(lib):
    for bits in (32, 8):
        g = _gen(9)
        ts = [_make(n, g, bits=bits) for n in (100, 5000)]
        here = _clone(ts)
        for t in (1, 2, 999, 123456):
            _run(lib, ts, 3e-4, t)
            _run(lib, here, torch.tensor([3e-4], device="cuda"), torch.tensor([t], device="cuda"))
            for a, b in zip(ts, here):
                # 1 / (1 - b^t) is rounded from 64 bits on both sides: at most a last bit apart
                assert (np.abs(f64(a["p"]) - f64(b["p"])) <= 4 * U * np.abs(f64(a["p"]))).all()
            assert _same([{k: t[k] for k in ("m", "v")} for t in ts], [{k: t[k] for k in ("m", "v")} for t in here])
    x = _lists(ts)
    for bad in (dict(lr=torch.tensor([1e-3])), dict(lr=torch.tensor([1e-3], device="cuda", dtype=torch.float64)),
                dict(step=torch.tensor([1, 2], device="cuda")), dict(step=torch.tensor([1.0], device="cuda")),
                dict(grad_scale=torch.ones(2, device="cuda"))):
        kw = dict(lr=1e-3, step=1)
        kw.update(bad)
        with pytest.raises(lib.LlamarlError):
            lib.adamw_step(x["p"], x["g"], x["m"], x["v"], kw.pop("lr"), kw.pop("step"), exp_avg_scales=x["ms"], exp_avg_sq_scales=x["vs"], **kw)


def test_second_moments_in_8_bits_follow_their_gradients(lib):
    """Gradients of constant size: v approaches their square though each step moves it by less than half a rounding step.
    After t steps v = g^2 (1 - b2^t); the mean over n entries of independently rounded roots is good to 3 in a hundred of that (a step is at most
    an eighth, the errors of a hundred steps add up to a few of them, and they are averaged over 4096 blocks)."""
    n = 1 << 19
    t = _make(n, _gen(10), bits=8, fresh=True)
    size = torch.where(torch.arange(n, device="cuda") % BLOCK == 0, 1.0, 0.37)      # a leading entry holds the block's factor
    t["g"].copy_(1e-3 * size)
    steps = 300
    for s in range(1, steps + 1):
        _run(lib, [t], 0.0, s)
    r = torch.from_numpy(np.sqrt(_held(t, "v")))
    want = 0.37e-3 * (1 - 0.999 ** steps) ** 0.5
    rest = r[(torch.arange(n) % BLOCK) != 0]
    assert abs(float(rest.mean()) / want - 1) < 0.03
    assert abs(float(r[::BLOCK].mean()) / (1e-3 * (1 - 0.999 ** steps) ** 0.5) - 1) < 1e-4      # tracked by the factor itself


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_of_all_gradients(lib, dtype):
    g = _gen(11)
    ts = [(torch.randn(n + 1, generator=g, device="cuda") * 10.0 ** (i % 5 - 2)).to(dtype)[i % 2:][:n] for i, n in enumerate(SIZES * 9)]
    want = np.sqrt(sum((f64(t) ** 2).sum() for t in ts))
    for max_norm in (0.5 * want, 2 * want, float("inf")):
        norm, scale = lib.grad_norm(ts, max_norm)
        assert abs(float(norm) - want) <= 1.01 * U * want
        assert abs(float(scale) - min(1.0, float(np.float32(max_norm)) / want)) <= 2 * U
    one, _ = lib.grad_norm([ts[-1]], 1.0)
    both, _ = lib.grad_norm([ts[-1], ts[-1]], 1.0)                         # listed twice: counted twice
    assert abs(float(both) / float(one) - 2 ** 0.5) < 1e-6


def test_norm_of_values_whose_squares_leave_fp32(lib):
    for size in (1e30, 1e-30):
        t = torch.full((100000,), size, device="cuda")
        norm, scale = lib.grad_norm([t], 1.0)
        assert abs(float(norm) / (size * 100000 ** 0.5) - 1) < 1e-6
        assert abs(float(scale) - min(1.0, 1 / (size * 100000 ** 0.5))) <= 2 * U
    for bad in (float("nan"), float("inf")):
        t = torch.ones(5000, device="cuda")
        t[4321] = bad
        norm, scale = lib.grad_norm([torch.ones(3, device="cuda"), t], 1.0)
        assert not np.isfinite(float(norm)) and np.isnan(float(scale))
    norm, scale = lib.grad_norm([torch.zeros(0, device="cuda"), torch.zeros(10, device="cuda")], 1.0)
    assert float(norm) == 0 and float(scale) == 1


def test_norm_and_step_replayed_from_a_graph(lib):
    """with step and rate on the device a captured pair takes the next step at every replay"""
    g = _gen(12)
    kinds = [dict(bits=8, param=torch.bfloat16, master=True), dict(bits=32)]
    ts = [_make(n, g, **kinds[i % 2]) for i, n in enumerate((100, 3001, 128, 40000))]
    eager = _clone(ts)
    grads = [[torch.randn_like(t["g"]) * 1e-2 for t in ts] for _ in range(4)]
    step, lr = torch.ones(1, dtype=torch.int64, device="cuda"), torch.zeros(1, device="cuda")
    ws = torch.empty(lib.grad_norm_workspace_bytes(len(ts)), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()

    def both(x):
        _, scale = lib.grad_norm([t["g"] for t in x], 0.3, ws=ws)
        _run(lib, x, lr, step, grad_scale=scale)

    warm = _clone(ts)
    with torch.cuda.stream(side):
        both(warm)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both(ts)
    torch.cuda.synchronize()
    assert _same(ts, eager)                                                # nothing ran yet
    for i, new in enumerate(grads):
        step.fill_(i + 1)
        lr.fill_(1e-3 / (i + 1))
        for x in (ts, eager):
            for t, n in zip(x, new):
                t["g"].copy_(n)
        torch.cuda.synchronize()
        ws.fill_(0xA5)
        graph.replay()
        torch.cuda.synchronize()
        both(eager)
        torch.cuda.synchronize()
        assert _same(ts, eager), i


def test_on_a_stream_of_its_own(lib):
    g = _gen(13)
    ts = [_make(n, g, bits=b) for n in (5000, 129) for b in (8, 32)]
    here = _clone(ts)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    norm, scale = lib.grad_norm([t["g"] for t in ts], 0.1, stream=side)
    _run(lib, ts, 1e-3, 2, grad_scale=scale, stream=side)
    side.synchronize()
    _, scale = lib.grad_norm([t["g"] for t in here], 0.1)
    _run(lib, here, 1e-3, 2, grad_scale=scale)
    torch.cuda.synchronize()
    assert _same(ts, here)


def test_list_arguments_are_checked(lib):
    t = _make(300, _gen(14), bits=8)
    f = torch.zeros(300, device="cuda")
    ok = dict(params=[t["p"]], grads=[t["g"]], exp_avgs=[t["m"]], exp_avg_sqs=[t["v"]], exp_avg_scales=[t["ms"]], exp_avg_sq_scales=[t["vs"]])
    for bad in (dict(exp_avgs=[f]), dict(exp_avg_sqs=[f]), dict(exp_avg_scales=None), dict(exp_avg_scales=[t["ms"][:2]]),
                dict(exp_avg_sq_scales=[t["vs"].double()]), dict(grads=[f[:299]]), dict(grads=[f.double()]), dict(params=[f.half()]),
                dict(params=[torch.zeros(300, 2, device="cuda")[:, 0]]), dict(grads=[f.cpu()]), dict(masters=[f]),
                dict(params=[t["p"].to(torch.bfloat16)], masters=[f.double()]), dict(params=[t["p"], t["p"]]),
                dict(exp_avgs=[t["v"]])):
        with pytest.raises(lib.LlamarlError):
            lib.adamw_step(lr=1e-3, step=1, **{**ok, **bad})
    v = t["p"]._version
    lib.adamw_step(lr=1e-3, step=1, **ok)
    assert t["p"]._version > v and t["m"]._version > 0


class TestOptimiser:
    def _model(self, dtype, seed=1):
        g = _gen(seed)
        shapes = [(33, 20), (257,), (128, 64), ()]
        return [torch.nn.Parameter((0.1 * torch.randn(s, generator=g, device="cuda")).to(dtype)) for s in shapes]

    def _gradients(self, ps, seed):
        g = _gen(seed)
        for p in ps:
            p.grad = (torch.randn(p.shape, generator=g, device="cuda") * 1e-2).to(p.dtype)

    def test_fp32_against_64_bits(self, lib):
        from paper_2505_24034_amd.optim import AdamW
        ps = self._model(torch.float32)
        ref = [f64(p) for p in ps]
        m, v = [np.zeros_like(r) for r in ref], [np.zeros_like(r) for r in ref]
        opt = AdamW([dict(params=ps[:2], lr=1e-2), dict(params=ps[2:], weight_decay=0.0)], lr=1e-3, max_grad_norm=0.2)
        for t in range(1, 6):
            self._gradients(ps, t)
            norm = np.sqrt(sum((f64(p.grad) ** 2).sum() for p in ps))
            opt.step()
            assert abs(float(opt.grad_norm) / norm - 1) < 1e-6
            for i, p in enumerate(ps):
                lr, wd = (1e-2, 0.01) if i < 2 else (1e-3, 0.0)
                ref[i], m[i], v[i] = adamw(ref[i], f64(p.grad), m[i], v[i], lr, t, 0.9, 0.999, 1e-8, wd, min(1.0, 0.2 / norm))
                # five steps of at most lr each, every one within 40 u of itself, and a rounding a step
                assert (np.abs(f64(p) - ref[i]) <= t * (40 * U * lr + U * (np.abs(ref[i]) + lr))).all()

    @pytest.mark.parametrize("bits", [8, 32])
    def test_saved_and_loaded_it_goes_on_alike(self, lib, bits):
        from paper_2505_24034_amd.optim import AdamW
        ps = self._model(torch.bfloat16)
        opt = AdamW(ps, lr=1e-2, state_bits=bits, max_grad_norm=1.0)
        for t in range(3):
            self._gradients(ps, t)
            opt.step()
        qs = [torch.nn.Parameter(p.detach().clone()) for p in ps]
        other = AdamW(qs, lr=1e-2, state_bits=bits, max_grad_norm=1.0)
        other.load_state_dict(opt.state_dict())
        for p, q in zip(ps, qs):
            for k, x in opt.state[p].items():
                y = other.state[q][k]
                assert (x.dtype == y.dtype and x.data_ptr() != y.data_ptr()) if torch.is_tensor(x) else x == y
        for t in range(3, 6):
            for x, o in ((ps, opt), (qs, other)):
                self._gradients(x, t)
                o.step()
        for p, q in zip(ps, qs):
            assert torch.equal(p, q) and torch.equal(opt.state[p]["master"], other.state[q]["master"])
            assert torch.equal(p, opt.state[p]["master"].to(torch.bfloat16))

    def test_parameters_without_a_gradient_and_steps_that_are_not_taken(self, lib):
        from paper_2505_24034_amd.optim import AdamW
        ps = self._model(torch.float32)
        opt = AdamW(ps, lr=1e-2, max_grad_norm=1.0)
        self._gradients(ps, 1)
        ps[0].grad = None
        before = [p.detach().clone() for p in ps]
        opt.step()
        assert torch.equal(ps[0], before[0]) and not torch.equal(ps[1], before[1]) and "step" not in opt.state[ps[0]]
        self._gradients(ps, 2)
        opt.step()                                                         # the first parameter is a step behind the others
        assert opt.state[ps[0]]["step"] == 1 and opt.state[ps[1]]["step"] == 2
        before = [p.detach().clone() for p in ps]
        ps[2].grad[3, 4] = float("inf")
        opt.step()
        assert all(torch.equal(p, b) for p, b in zip(ps, before))
        ps[2].grad = torch.randn(64, 128, device="cuda").T                 # a gradient in another order than its parameter
        opt.step()
        assert torch.isfinite(ps[2]).all() and not torch.equal(ps[2], before[2])

    def test_rate_as_a_tensor(self, lib):
        from paper_2505_24034_amd.optim import AdamW
        for rate in (torch.tensor(1e-2), torch.tensor([1e-2], device="cuda")):
            ps, qs = self._model(torch.float32), self._model(torch.float32)
            a, b = AdamW(ps, lr=float(torch.tensor(1e-2))), AdamW(qs, lr=rate)
            for t in range(2):
                for x, o in ((ps, a), (qs, b)):
                    self._gradients(x, t)
                    o.step()
            assert all(torch.equal(p, q) for p, q in zip(ps, qs))

    def test_goes_on_from_torchs_states(self, lib):
        from paper_2505_24034_amd.optim import AdamW
        ps, qs = self._model(torch.float32), self._model(torch.float32)
        theirs, ours = torch.optim.AdamW(ps, lr=1e-2, weight_decay=0.1), AdamW(qs, lr=1e-2, weight_decay=0.1)
        for t in range(4):
            if t == 2:
                for p, q in zip(ps, qs):
                    q.data.copy_(p.data)
                ours.load_state_dict(theirs.state_dict())
            self._gradients(ps, t)
            theirs.step()
            if t >= 2:
                self._gradients(qs, t)
                ours.step()
        for p, q in zip(ps, qs):
            # two steps of at most 1.1 lr each, every one within 40 u of itself on either side, and two roundings a step
            assert (np.abs(f64(p) - f64(q)) <= 2 * (80 * U * 1.1e-2 + 2 * U * (np.abs(f64(p)) + 1.1e-2))).all()
            assert ours.state[q]["step"] == 4
