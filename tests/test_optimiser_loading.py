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
