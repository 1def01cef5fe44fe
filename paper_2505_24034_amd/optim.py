"""AdamW as a torch optimiser over the library's kernels: `llamarl_grad_norm` and `llamarl_adamw_step` in include/llamarl.h.  A
launch for every 48 tensors, another and one more where the norm is asked for; nothing waits for the device, and no arithmetic
happens here."""
import torch

from . import binding as L


class AdamW(torch.optim.Optimizer):
    """params: contiguous float32 or bfloat16 tensors on the GPU, or groups of them.

    state_bits      32, or 8: a quarter of the memory (binding.adamw_step says how they are held); betas[0] is then 15/16 at most
    master_weights  keep a float32 copy of bfloat16 parameters, which is what moves; without it changes below half a
                    parameter's last bit are lost.  It is taken at the parameter's first step, or the first behind a load of states
                    without one: weights that are loaded later have to come with the optimiser's state
    max_grad_norm   scale the gradients of all groups down to this norm; `grad_norm` then holds the norm before it (one
                    element, on the device).  A norm that is not finite leaves every parameter and state as it was (the step is
                    counted); without max_grad_norm nothing looks for such gradients

    lr, betas, eps, weight_decay are read from the groups at every step, as schedulers set them; lr may be a tensor (one on the
    GPU is read there, when the kernels run).  Groups of torch.optim.Adam and AdamW with amsgrad, maximize or a decay inside the
    gradient are refused."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, state_bits=32, master_weights=True,
                 max_grad_norm=None):
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32 (got %r)" % (state_bits,))
        self.state_bits, self.master_weights, self.max_grad_norm, self.grad_norm = state_bits, master_weights, max_grad_norm, None
        super().__init__(params, dict(lr=lr, betas=betas, eps=eps, weight_decay=weight_decay))

    def __getstate__(self):
        """As torch's, which would leave out what it does not know."""
        own = ("state_bits", "master_weights", "max_grad_norm", "grad_norm")
        return {**super().__getstate__(), **{name: getattr(self, name) for name in own}}

    def add_param_group(self, param_group):
        self._check_group(param_group)
        super().add_param_group(param_group)

    def _check_group(self, group):
        """torch's settings that change the step and are not computed here, and what states in 8 bits cannot follow"""
        beta1 = group.get("betas", self.defaults["betas"])[0]
        if self.state_bits == 8 and beta1 > L.STATE_BETA1:
            raise L.LlamarlError(L.ERR_INVALID_ARG, "first moments in 8 bits need betas[0] <= %g (got %g)" % (L.STATE_BETA1, beta1))
        set_ = [name for name in ("amsgrad", "maximize") if group.get(name)]
        if not group.get("decoupled_weight_decay", True) and group.get("weight_decay", self.defaults["weight_decay"]):
            set_.append("decoupled_weight_decay=False")
        if set_:
            raise L.LlamarlError(L.ERR_UNSUPPORTED, "a parameter group with " + ", ".join(set_))

    def _init_state(self, p):
        s = self.state[p]
        n = p.numel()
        s["step"] = 0
        if self.state_bits == 8:
            blocks = -(-n // L.STATE_BLOCK)
            for name in ("exp_avg", "exp_avg_sq"):
                s[name] = torch.zeros(p.shape, dtype=torch.uint8, device=p.device).view(torch.float8_e4m3fn)
                s[name + "_scale"] = torch.zeros(blocks, device=p.device)
        else:
            for name in ("exp_avg", "exp_avg_sq"):
                s[name] = torch.zeros(p.shape, device=p.device)
        return s

    def _has_master(self, p):
        return self.master_weights and p.dtype == torch.bfloat16

    @torch.no_grad()
    def step(self, closure=None):
        """One step for every parameter that has a gradient."""
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        if torch.cuda.is_available() and torch.cuda.is_current_stream_capturing():
            raise L.LlamarlError(L.ERR_UNSUPPORTED, "a captured step would repeat its step count: capture binding.adamw_step "
                                                    "with step and lr on the device")
        runs = {}                                         # (group, step) -> parameters and gradients
        for group in self.param_groups:                   # before any of them moves
            self._check_group(group)
        for i, group in enumerate(self.param_groups):
            for p in group["params"]:
                if p.grad is None:
                    continue
                if p.grad.is_sparse:
                    raise L.LlamarlError(L.ERR_UNSUPPORTED, "sparse gradients")
                s = self.state[p] if self.state[p] else self._init_state(p)
                if self._has_master(p) and "master" not in s:
                    s["master"] = p.detach().float()
                runs.setdefault((i, s["step"] + 1), []).append((p, p.grad.contiguous()))
        if not runs:
            return loss
        scale = None
        if self.max_grad_norm is not None:
            self.grad_norm, scale = L.grad_norm([g for pairs in runs.values() for _, g in pairs], self.max_grad_norm)
        for (i, step), pairs in runs.items():
            group, states = self.param_groups[i], [self.state[p] for p, _ in pairs]
            lr = group["lr"]
            if torch.is_tensor(lr) and not lr.is_cuda:
                lr = float(lr)
            def column(name):
                return [s.get(name) for s in states]
            L.adamw_step([p for p, _ in pairs], [g for _, g in pairs], column("exp_avg"), column("exp_avg_sq"), lr, step,
                         betas=group["betas"], eps=group["eps"], weight_decay=group["weight_decay"], masters=column("master"),
                         exp_avg_scales=column("exp_avg_scale"), exp_avg_sq_scales=column("exp_avg_sq_scale"), grad_scale=scale)
            for s in states:
                s["step"] = step
        return loss

    def load_state_dict(self, state_dict):
        """As torch's, which would turn the states into the parameters' type.  float32 states of torch.optim.AdamW can be gone on from
        with state_bits=32; states of another type than state_bits asks for are refused.  Master copies are taken where this
        optimiser keeps them."""
        seen = []                                         # what torch takes: its hooks may have made another one of state_dict

        def check(_, taken):
            for group in taken["param_groups"]:
                self._check_group(group)
            for k, p in self._saved_places(taken):
                if taken["state"].get(k):
                    self._check_state(p, taken["state"][k])
            seen.append(taken)

        handles = [self.register_load_state_dict_pre_hook(check),                                    # behind all others
                   self.register_load_state_dict_post_hook(lambda _: self._take(seen[0]), prepend=True)]      # ahead of them
        try:
            super().load_state_dict(state_dict)
        finally:
            for h in handles:
                h.remove()

    def _saved_places(self, state_dict):
        """(key of a saved state, parameter)"""
        saved = [k for group in state_dict["param_groups"] for k in group["params"]]
        return zip(saved, [p for group in self.param_groups for p in group["params"]])

    def _check_state(self, p, s):
        want = dict.fromkeys(("exp_avg", "exp_avg_sq"), (torch.float8_e4m3fn if self.state_bits == 8 else torch.float32, p.numel()))
        if self.state_bits == 8:
            want.update(dict.fromkeys(("exp_avg_scale", "exp_avg_sq_scale"), (torch.float32, -(-p.numel() // L.STATE_BLOCK))))
        if self._has_master(p) and "master" in s:
            want["master"] = (torch.float32, p.numel())
        for name, (dtype, n) in want.items():
            x = s.get(name)
            if not torch.is_tensor(x) or x.dtype != dtype or x.numel() != n:
                raise L.LlamarlError(L.ERR_INVALID_ARG, "saved states with %s of %s; state_bits=%d takes %d entries of %s here" % (
                    name, "%d entries of %s" % (x.numel(), x.dtype) if torch.is_tensor(x) else type(x).__name__, self.state_bits, n, dtype))

    def _take(self, state_dict):
        for k, p in self._saved_places(state_dict):
            if k in state_dict["state"]:
                self.state[p] = {name: int(v) if name == "step" else v.detach().to(p.device, copy=True) if torch.is_tensor(v) else v
                                 for name, v in state_dict["state"][k].items() if name != "master" or self._has_master(p)}
