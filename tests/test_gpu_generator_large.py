"""Arrays of more than 2^31 entries: offsets of the last rows do not wrap.  The last rows of a large call are those of a small one, bit for bit."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _free():
    torch.cuda.empty_cache()


def test_norm_and_its_quantised_outputs(lib):
    N, d, k = 131200, 16384, 5
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(N, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    w = torch.rand(d, device="cuda", generator=g) + 0.5
    assert x.numel() > 1 << 31
    h, s, rstd = lib.rms_norm(x, w, 1e-5, residual=x)
    hk, sk, rk = lib.rms_norm(x[-k:].contiguous(), w, 1e-5, residual=x[-k:].contiguous())
    assert torch.equal(h[-k:], hk) and torch.equal(s[-k:], sk) and torch.equal(rstd[-k:], rk)
    dx, dw = lib.rms_norm_bwd(h, s, w, rstd, dsum=x, dweight_dtype=torch.float32)
    dxk, _ = lib.rms_norm_bwd(hk, sk, w, rk, dsum=x[-k:].contiguous(), dweight_dtype=torch.float32)
    assert torch.equal(dx[-k:], dxk)
    cols = slice(d - 3, d)
    want = (h[:, cols].double() * s[:, cols].double() * rstd.double()[:, None]).sum(dim=0)
    # every term is positive here (h = n w): a chain of fewer additions than rows of a workgroup, workgroups and slices, one rounding each
    assert ((dw[cols].double() / want - 1).abs() < (N // 256 + 300) * 2.0 ** -24).all()
    del dx, h
    _free()
    for call in (lib.rms_norm_rows, lib.rms_norm_blocks):
        q, scale, _ = call(x, w, 1e-5)
        qk, scale_k, _ = call(x[-k:].contiguous(), w, 1e-5)
        assert torch.equal(q[-k:].view(torch.uint8), qk.view(torch.uint8))
        at = scale[-k:] if scale.dim() == 1 else scale.view(torch.uint8)[:, -k:]
        assert torch.equal(at, scale_k if scale.dim() == 1 else scale_k.view(torch.uint8))
    q, scale = lib.quantise_rows(x)
    qk, scale_k = lib.quantise_rows(x[-k:].contiguous())
    assert torch.equal(q[-k:], qk) and torch.equal(scale[-k:], scale_k)
    _free()


def test_logits_and_head_of_more_than_2_to_the_31(lib):
    g = torch.Generator(device="cuda").manual_seed(2)
    i8 = lambda *s: torch.randint(-127, 128, s, dtype=torch.int8, device="cuda", generator=g)  # noqa: E731
    N, V, d = 17000, 128256, 64
    H, W, hs, ws = i8(N, d), i8(V, d), torch.rand(N, device="cuda", generator=g), torch.rand(V, device="cuda", generator=g)
    z = lib.logits_rows(H, hs, W, ws)
    assert z.numel() > 1 << 31
    assert torch.equal(z[-3:], lib.logits_rows(H[-3:].contiguous(), hs[-3:].contiguous(), W, ws))
    del z
    _free()
    V, d = 17000, 131056                                                   # W alone
    W, ws = i8(V, d), torch.rand(V, device="cuda", generator=g)
    assert W.numel() > 1 << 31
    for N in (3, 40, 300):
        H, hs = i8(N, d), torch.rand(N, device="cuda", generator=g)
        z = lib.logits_rows(H, hs, W, ws)
        assert torch.equal(z[:, -70:], lib.logits_rows(H, hs, W[-70:].contiguous(), ws[-70:].contiguous()))
    _free()


def test_drafts_over_more_than_2_to_the_31_logits(lib):
    g = torch.Generator(device="cuda").manual_seed(3)
    B, K, V, k = 2200, 7, 128256, 3
    z = torch.empty(B, K + 1, V, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    y = torch.empty(B, K, V, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    z[:, :K] += y
    assert z.numel() > 1 << 31
    drafts = y.argmax(dim=2).to(torch.int32)
    u = torch.rand(B, K + 1, device="cuda", generator=g)
    got = lib.verify_drafts(z, drafts, u, draft_logits=y)
    c = lambda t: t[-k:].contiguous()  # noqa: E731
    want = lib.verify_drafts(c(z), c(drafts), c(u), draft_logits=c(y))
    assert all(torch.equal(a[-k:], b) for a, b in zip(got, want))
    _free()
