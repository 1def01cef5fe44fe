"""What `optim.AdamW` takes from a checkpoint, and what it refuses: no kernel runs."""
import copy

import pytest
import torch

from paper_2505_24034_amd import binding as L
from paper_2505_24034_amd.optim import AdamW


def _params(dtype=torch.float32):
    g = torch.Generator().manual_seed(1)
    return [torch.nn.Parameter(torch.randn(s, generator=g).to(dtype)) for s in ((3, 5), (7,))]


def _saved(cls=torch.optim.AdamW, dtype=torch.float32, steps=2, **kw):
    """the state_dict of one of torch's optimisers after some steps"""
    ps = _params(dtype)
    opt = cls(ps, lr=1e-2, **kw)
    for _ in range(steps):
        for p in ps:
            p.grad = torch.ones_like(p)
        opt.step()
    return opt.state_dict()


@pytest.mark.parametrize("cls,kw,names", [(torch.optim.AdamW, dict(maximize=True), ["maximize"]), (torch.optim.AdamW, dict(amsgrad=True), ["amsgrad"]),
                                          (torch.optim.AdamW, dict(amsgrad=True, maximize=True), ["amsgrad", "maximize"]),
                                          (torch.optim.Adam, dict(weight_decay=0.1), ["decoupled_weight_decay"])])
def test_settings_that_are_not_followed_are_refused(cls, kw, names):
    opt = AdamW(_params(), lr=1e-3)
    before = copy.deepcopy(opt.state_dict())
    with pytest.raises(L.LlamarlError) as e:
        opt.load_state_dict(_saved(cls, **kw))
    assert all(n in str(e.value) for n in names)
    assert opt.state_dict() == before                                      # nothing was taken
    if cls is torch.optim.AdamW:                                           # nor through a group's own settings
        with pytest.raises(L.LlamarlError):
            AdamW([dict(params=_params(), **kw)], lr=1e-3)


@pytest.mark.parametrize("cls,kw", [(torch.optim.AdamW, dict(weight_decay=0.1)), (torch.optim.Adam, dict())])
def test_settings_that_are_followed_are_taken(cls, kw):
    opt = AdamW(_params(), lr=1e-3)
    saved = _saved(cls, betas=(0.8, 0.9), eps=1e-6, **kw)
    opt.load_state_dict(saved)
    g = opt.param_groups[0]
    assert (g["lr"], g["betas"], g["eps"], g["weight_decay"]) == (1e-2, (0.8, 0.9), 1e-6, kw.get("weight_decay", 0))
    for i, p in enumerate(g["params"]):
        s = opt.state[p]
        assert s["step"] == 2 and isinstance(s["step"], int)
        for name in ("exp_avg", "exp_avg_sq"):
            assert torch.equal(s[name], saved["state"][i][name]) and s[name].data_ptr() != saved["state"][i][name].data_ptr()


def test_hooks_of_a_load_see_and_change_what_is_taken():
    """the dict that a hook before the load returns is the one that is taken, and a hook behind it finds the states in place"""
    saved = _saved()
    renamed = dict(saved, state={i + 1: s for i, s in saved["state"].items()}, param_groups=[dict(saved["param_groups"][0], params=[1, 2])])
    untouched = copy.deepcopy(renamed)
    opt = AdamW(_params(), lr=1e-3)

    def before(o, d):
        assert o is opt
        return dict(d, state={k: dict(s, exp_avg=s["exp_avg"] * 2, step=7) for k, s in d["state"].items()})

    def behind(o):
        for s in o.state.values():
            assert s["step"] == 7 and isinstance(s["step"], int)
            s["exp_avg"] += 1

    opt.register_load_state_dict_pre_hook(before)
    opt.register_load_state_dict_post_hook(behind)
    for _ in range(2):                                                     # a load leaves no hook of its own behind
        opt.load_state_dict(renamed)
        for i, p in enumerate(opt.param_groups[0]["params"]):
            assert torch.equal(opt.state[p]["exp_avg"], saved["state"][i]["exp_avg"] * 2 + 1)
    for i in (1, 2):
        assert torch.equal(renamed["state"][i]["exp_avg"], untouched["state"][i]["exp_avg"])


def test_settings_that_a_hook_brings_are_looked_at():
    opt = AdamW(_params(), lr=1e-3)
    opt.register_load_state_dict_pre_hook(lambda o, d: dict(d, param_groups=[dict(g, maximize=True) for g in d["param_groups"]]))
    with pytest.raises(L.LlamarlError):
        opt.load_state_dict(_saved())
    assert not opt.state


def _own(bits, dtype, master):
    """(optimiser, its state as a step would have left it) without a step"""
    opt = AdamW(_params(dtype), lr=1e-3, state_bits=bits, master_weights=master)
    for p in opt.param_groups[0]["params"]:
        s = opt._init_state(p)
        s["step"] = 3
        if master and dtype == torch.bfloat16:
            s["master"] = p.detach().float() + 2.0 ** -12
    return opt


@pytest.mark.parametrize("bits", [8, 32])
def test_states_of_other_bits_are_refused(bits):
    opt = AdamW(_params(), lr=1e-3, state_bits=bits)
    with pytest.raises(L.LlamarlError, match="state_bits=%d" % bits):
        opt.load_state_dict(_own(40 - bits, torch.float32, True).state_dict())
    assert not opt.state
    if bits == 8:                                                          # torch's own are in 32 bits
        with pytest.raises(L.LlamarlError, match="state_bits=8"):
            opt.load_state_dict(_saved())
    for drop in ("exp_avg", "exp_avg_sq") + (("exp_avg_scale", "exp_avg_sq_scale") if bits == 8 else ()):
        saved = _own(bits, torch.float32, True).state_dict()
        for s in saved["state"].values():
            s[drop] = s[drop].view(torch.uint8)[:2].view(s[drop].dtype) if s[drop].dtype == torch.float8_e4m3fn else s[drop].reshape(-1)[:0]
        with pytest.raises(L.LlamarlError, match=drop):
            opt.load_state_dict(saved)
    with pytest.raises(L.LlamarlError, match="bfloat16"):                  # torch keeps bf16 parameters' states in bf16
        AdamW(_params(torch.bfloat16), lr=1e-3).load_state_dict(_saved(dtype=torch.bfloat16))
    opt.load_state_dict(_own(bits, torch.float32, True).state_dict())
    assert all(s["step"] == 3 for s in opt.state.values())


def test_master_copies_are_there_where_they_are_asked_for(monkeypatch):
    calls = []
    monkeypatch.setattr(L, "adamw_step", lambda params, *a, **kw: calls.append((params, kw["masters"])))
    for saved_master in (True, False):
        for master in (True, False):
            saved = _own(32, torch.bfloat16, saved_master).state_dict()
            opt = AdamW(_params(torch.bfloat16), lr=1e-3, master_weights=master)
            opt.load_state_dict(saved)
            ps = opt.param_groups[0]["params"]
            with torch.no_grad():
                for p in ps:
                    p += 1                                                 # weights that are loaded behind the states
                    p.grad = torch.ones_like(p)
            opt.step()
            params, masters = calls.pop()
            assert all(a is b for a, b in zip(params, ps))
            for i, (p, m) in enumerate(zip(ps, masters)):
                if not master:
                    assert m is None
                elif saved_master:
                    assert torch.equal(m, saved["state"][i]["master"]) and m.data_ptr() != saved["state"][i]["master"].data_ptr()
                else:
                    assert m.dtype == torch.float32 and torch.equal(m, p.detach().float())
    opt = AdamW(_params(torch.float32), lr=1e-3)                           # float32 parameters have none
    opt.load_state_dict(_own(32, torch.bfloat16, True).state_dict())
    assert all("master" not in s for s in opt.state.values())
