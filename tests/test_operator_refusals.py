"""What the optimiser step and the 8-bit head refuse, without a GPU: every check comes before anything is launched."""
import copy
import ctypes

import pytest
import torch

from paper_2505_24034_amd import binding as L
from paper_2505_24034_amd.optim import AdamW

no_gpu_only = pytest.mark.skipif(torch.cuda.device_count() > 0, reason="fake device pointers: CPU-only test")
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def clib():
    return L.load()


def _tensor(at=1 << 24, n=1000, param_dt=L.F32, grad_dt=L.F32, bits8=False, **kw):
    """a tensor of made-up, disjoint device addresses"""
    step = 1 << 16
    f = dict(param=at, master=None, grad=at + step, m=at + 2 * step, v=at + 3 * step, m_scale=at + 4 * step if bits8 else None,
             v_scale=at + 5 * step if bits8 else None, n=n, param_dt=param_dt, grad_dt=grad_dt)
    f.update(kw)
    return L.AdamwTensor(**f)


def _adamw(clib, *tensors, scale=None, lr_device=None, step_device=None, count=None, **kw):
    p = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, step=1)
    p.update(kw)
    arr = (L.AdamwTensor * max(len(tensors), 1))(*tensors)
    return clib.llamarl_adamw_step(arr, len(tensors) if count is None else count, ctypes.byref(L.AdamwParams(**p)), scale, lr_device,
                                   step_device, None)


@no_gpu_only
@pytest.mark.parametrize("kw", [dict(lr=-1.0), dict(lr=NAN), dict(lr=INF), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=NAN), dict(beta2=1.0),
                                dict(eps=-1e-9), dict(eps=INF), dict(weight_decay=-0.1), dict(weight_decay=NAN), dict(step=0), dict(count=-1),
                                dict(scale=ctypes.c_void_p(2)), dict(lr_device=ctypes.c_void_p(6)), dict(step_device=ctypes.c_void_p(12))])
def test_adamw_refuses_hyperparameters(clib, kw):
    assert _adamw(clib, _tensor(), **kw) == L.ERR_INVALID_ARG
    assert clib.llamarl_last_error()


@no_gpu_only
@pytest.mark.parametrize("kw", [dict(n=-1), dict(param=None), dict(grad=None), dict(m=None), dict(v=None), dict(param_dt=2), dict(grad_dt=7),
                                dict(m_scale=1 << 30), dict(v_scale=1 << 30), dict(master=1 << 30), dict(param=(1 << 24) + 2),
                                dict(m=(1 << 25) + 2), dict(grad=(1 << 25) + 1, grad_dt=L.BF16)])
def test_adamw_refuses_tensors(clib, kw):
    assert _adamw(clib, _tensor(1 << 28), _tensor(**kw)) == L.ERR_INVALID_ARG
    assert b"tensor 1" in clib.llamarl_last_error()


@no_gpu_only
def test_adamw_refuses_what_overlaps(clib):
    a, b = _tensor(), _tensor(1 << 28)
    assert _adamw(clib, a, b, a) == L.ERR_INVALID_ARG and b"overlap" in clib.llamarl_last_error()
    # the last word of one array is the first of another, in either order
    for name in ("param", "grad", "m", "v"):
        for off in (999 * 4, -999 * 4):
            assert _adamw(clib, a, _tensor(1 << 28, **{name: a.param + off})) == L.ERR_INVALID_ARG, name
    # a long array that starts far before: not only neighbours in the order of addresses are compared
    long = _tensor(1 << 36, n=1 << 20, m=(1 << 24) - (1 << 21), grad=1 << 40)
    assert _adamw(clib, a, b, long) == L.ERR_INVALID_ARG
    s = _tensor(1 << 29, bits8=True)
    assert _adamw(clib, s, _tensor(1 << 30, m=s.v_scale + 7 * 4)) == L.ERR_INVALID_ARG      # eight factors for 1000 entries
    # gradients are only read: two tensors may share one, and nothing else may lie over it
    assert _adamw(clib, _tensor(), _tensor(1 << 28, grad=_tensor().m + 16)) == L.ERR_INVALID_ARG


@no_gpu_only
def test_sizes_that_no_launch_takes(clib):
    assert _adamw(clib, _tensor(n=1 << 39, grad=1 << 50, m=1 << 51, v=1 << 52, param=1 << 53)) == L.ERR_UNSUPPORTED
    g = (L.Gradient * 1)(L.Gradient(1 << 24, 1 << 39, L.F32))
    assert clib.llamarl_grad_norm(g, 1, 1.0, ctypes.c_void_p(64), ctypes.c_void_p(128), ctypes.c_void_p(256), 1 << 20, None) == L.ERR_UNSUPPORTED
    assert _adamw(clib, count=0) == L.OK                                   # nothing to do, and nothing done
    assert _adamw(clib, _tensor(n=0, param=None, grad=None, m=None, v=None)) == L.OK


@no_gpu_only
def test_grad_norm_refuses(clib):
    vp = ctypes.c_void_p

    def call(g=L.Gradient(1 << 24, 100, L.F32), count=1, max_norm=1.0, norm=1 << 10, scale=1 << 11, ws=1 << 12, ws_bytes=1 << 20):
        return clib.llamarl_grad_norm((L.Gradient * 1)(g), count, max_norm, vp(norm), vp(scale), vp(ws), ws_bytes, None)

    for bad in (dict(norm=None), dict(scale=None), dict(count=-1), dict(max_norm=0.0), dict(max_norm=NAN), dict(max_norm=-1.0),
                dict(g=L.Gradient(None, 100, L.F32)), dict(g=L.Gradient(1 << 24, -1, L.F32)), dict(g=L.Gradient(1 << 24, 1, 3)),
                dict(g=L.Gradient((1 << 24) + 2, 100, L.F32)), dict(ws=(1 << 12) + 8), dict(norm=6)):
        assert call(**bad) == L.ERR_INVALID_ARG, bad
    assert call(ws=None) == L.ERR_WORKSPACE and call(ws_bytes=L.grad_norm_workspace_bytes(1) - 1) == L.ERR_WORKSPACE
    assert L.grad_norm_workspace_bytes(-1) == 0 and L.grad_norm_workspace_bytes(0) > 0


@no_gpu_only
def test_quantise_refuses(clib):
    vp = ctypes.c_void_p

    def call(x=1 << 24, rows=10, cols=64, dt=L.BF16, block=1, q=1 << 26, scale=1 << 28):
        return clib.llamarl_quantise_blocks(vp(x), rows, cols, dt, block, vp(q), vp(scale), None)

    for bad in (dict(x=None), dict(q=None), dict(scale=None), dict(rows=0), dict(cols=0), dict(rows=-5), dict(dt=2), dict(block=0),
                dict(block=64), dict(x=(1 << 24) + 8), dict(q=(1 << 26) + 4), dict(scale=(1 << 28) + 1), dict(q=(1 << 24) + 16),
                dict(scale=1 << 24), dict(scale=(1 << 26) + 636)):
        assert call(**bad) == L.ERR_INVALID_ARG, bad
    for bad in (dict(cols=24), dict(cols=8), dict(cols=1 << 22), dict(rows=1 << 31)):
        assert call(**bad) == L.ERR_UNSUPPORTED, bad


@no_gpu_only
def test_head_products_refuse(clib):
    vp = ctypes.c_void_p

    def logits(H=1 << 24, Hs=1 << 25, W=1 << 26, Ws=1 << 27, N=10, d=64, V=50, dt=L.F32, z=1 << 28):
        return clib.llamarl_logits_blocks(vp(H), vp(Hs), vp(W), vp(Ws), N, d, V, dt, vp(z), None)

    def logprobs(H=1 << 24, Hs=1 << 25, W=1 << 26, Ws=1 << 27, N=10, d=64, V=50, tg=1 << 28, logp=1 << 29, lse=1 << 30, ws=1 << 31, ws_bytes=1 << 30):
        return clib.llamarl_token_logprobs_blocks(vp(H), vp(Hs), vp(W), vp(Ws), vp(tg), None, N, d, V, vp(logp), vp(lse), vp(ws), ws_bytes, None)

    for call in (logits, logprobs):
        for bad in (dict(H=None), dict(Hs=None), dict(W=None), dict(Ws=None), dict(N=0), dict(d=0), dict(V=0), dict(N=-1), dict(H=(1 << 24) + 8),
                    dict(W=(1 << 26) + 1), dict(Hs=(1 << 25) + 2), dict(Ws=(1 << 27) + 3)):
            assert call(**bad) == L.ERR_INVALID_ARG, bad
        for bad in (dict(d=72), dict(V=1 << 21), dict(N=1 << 26, d=64), dict(d=1 << 22)):
            assert call(**bad) == L.ERR_UNSUPPORTED, bad
    assert logits(z=None) == L.ERR_INVALID_ARG and logits(dt=5) == L.ERR_INVALID_ARG and logits(z=(1 << 28) + 4) == L.ERR_INVALID_ARG
    for bad in (dict(tg=None), dict(logp=None), dict(lse=None), dict(tg=(1 << 28) + 2), dict(ws=(1 << 31) + 4)):
        assert logprobs(**bad) == L.ERR_INVALID_ARG, bad
    assert logprobs(ws=None) == L.ERR_WORKSPACE
    assert logprobs(ws_bytes=L.logprobs_blocks_workspace_bytes(10, 50) - 1) == L.ERR_WORKSPACE


def test_logprobs_workspace_does_not_fall(clib):
    sizes = [1, 16, 31, 63, 64, 65, 100, 127, 128, 129, 255, 256, 1000, 5003, 16384]
    vocabs = [1, 31, 32, 33, 128, 1000, 12288, 49152, 128256]
    size = {(n, v): L.logprobs_blocks_workspace_bytes(n, v) for n in sizes for v in vocabs}
    for v in vocabs:
        assert all(size[a, v] <= size[b, v] for a, b in zip(sizes, sizes[1:]))
    for n in sizes:
        assert all(size[n, a] <= size[n, b] for a, b in zip(vocabs, vocabs[1:]))
    assert L.logprobs_blocks_workspace_bytes(0, 5) == L.logprobs_blocks_workspace_bytes(5, 0) == 0


def test_binding_refuses_what_is_not_on_the_device_or_of_the_type(clib):
    f, b = torch.zeros(8), torch.zeros(8, dtype=torch.bfloat16)
    with pytest.raises(L.LlamarlError, match="device"):
        L.grad_norm([f], 1.0)
    with pytest.raises(L.LlamarlError, match="at least one"):
        L.grad_norm([], 1.0)
    with pytest.raises(TypeError):
        L.grad_norm([None], 1.0)
    with pytest.raises(TypeError):
        L.grad_norm(5, 1.0)
    with pytest.raises(L.LlamarlError, match="device"):
        L.adamw_step([f], [f], [f], [f], 1e-3, 1)
    with pytest.raises(L.LlamarlError, match="grads must have 1"):
        L.adamw_step([f], [], [f], [f], 1e-3, 1)
    with pytest.raises(L.LlamarlError, match="masters must have 1"):
        L.adamw_step([f], [f], [f], [f], 1e-3, 1, masters=[])
    L.adamw_step([], [], [], [], 1e-3, 1)
    for call in (lambda: L.quantise_blocks(f.view(1, 8), 1), lambda: L.quantise_blocks(b.view(1, 8), 128)):
        with pytest.raises(L.LlamarlError, match="device"):
            call()
    q, s = torch.zeros(2, 16, dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros(1, 2, 4, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    with pytest.raises(L.LlamarlError, match="H must be"):
        L.logits_blocks(q, s, q, s)
    with pytest.raises(L.LlamarlError, match="H must be"):
        L.token_logprobs_blocks(q, s, q, s, torch.zeros(2, dtype=torch.int32))


def test_optimiser_refuses():
    p = torch.nn.Parameter(torch.zeros(4))
    with pytest.raises(ValueError):
        AdamW([p], state_bits=16)
    assert AdamW([p]).step() is None                                       # no gradient: nothing to do


@no_gpu_only
def test_outputs_do_not_lie_over_operands(clib):
    vp = ctypes.c_void_p
    a = _tensor()
    for kw in (dict(scale=vp(a.param + 996 * 4 + 12)), dict(lr_device=vp(a.v)), dict(step_device=vp(a.m + 8))):
        assert _adamw(clib, _tensor(1 << 28), a, **kw) == L.ERR_INVALID_ARG
        assert b"lies in tensor 1" in clib.llamarl_last_error()
    g = (L.Gradient * 2)(L.Gradient(1 << 20, 10, L.BF16), L.Gradient(1 << 24, 100, L.F32))
    for norm, scale, ws in ((1 << 10, 1 << 10, 1 << 12), (1 << 10, 1 << 12, 1 << 12), ((1 << 24) + 396, 1 << 11, 1 << 12),
                            (1 << 10, (1 << 20) + 16, 1 << 12), (1 << 10, 1 << 11, (1 << 24) - 16)):
        assert clib.llamarl_grad_norm(g, 2, 1.0, vp(norm), vp(scale), vp(ws), 1 << 20, None) == L.ERR_INVALID_ARG
        assert b"norm" in clib.llamarl_last_error()
    H, Hs, W, Ws, N, d, V = 1 << 24, 1 << 25, 1 << 26, 1 << 27, 10, 64, 50
    for z in (H, H + 624, Hs + 32, W - 16, W + 50 * 64 - 16, Ws):
        assert clib.llamarl_logits_blocks(vp(H), vp(Hs), vp(W), vp(Ws), N, d, V, L.F32, vp(z), None) == L.ERR_INVALID_ARG
        assert b"overlap" in clib.llamarl_last_error()
    tg, mask = 1 << 28, 1 << 29
    for logp, lse, ws in ((1 << 30, 1 << 30, 1 << 31), (tg + 36, 1 << 30, 1 << 31), (1 << 30, mask + 8, 1 << 31), (1 << 30, 1 << 32, 1 << 30),
                          (1 << 30, 1 << 32, W)):
        assert clib.llamarl_token_logprobs_blocks(vp(H), vp(Hs), vp(W), vp(Ws), vp(tg), vp(mask), N, d, V, vp(logp), vp(lse), vp(ws), 1 << 20,
                                                  None) == L.ERR_INVALID_ARG
        assert b"overlap" in clib.llamarl_last_error()


def test_optimiser_is_copied_whole():
    opt = AdamW([torch.nn.Parameter(torch.zeros(4))], state_bits=8, master_weights=False, max_grad_norm=2.0)
    twin = copy.deepcopy(opt)
    assert (twin.state_bits, twin.master_weights, twin.max_grad_norm, twin.grad_norm) == (8, False, 2.0, None)
    assert twin.step() is None
