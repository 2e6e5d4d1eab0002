"""AdamW as a torch optimiser around dpb_adamw_step: every parameter of one
dtype in one launch, states in 32 bits or in 8.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import dpb


class AdamW(torch.optim.Optimizer):
    """AdamW with decoupled weight decay over fp32 and bf16 parameters.

    ``state_bits`` 32: fp32 moments. 8: e4m3 codes with a scale for each 256
    values, stored with stochastic rounding drawn from ``seed`` (kept in the
    parameter groups, so in state_dict()) and the step (2 bytes a parameter in
    place of 8). ``step(grad_scale=...)`` takes a
    device tensor that multiplies the gradients; where it is not finite, no
    parameter or state changes (the step still counts). A step's number and
    what follows from it (bias corrections, random bits) come from the host,
    so a step cannot be captured into a CUDA graph."""

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 1e-2,
                 state_bits: int = 32, seed: int = 0):
        if state_bits not in (32, 8):
            raise ValueError("state_bits must be 32 or 8")
        self._sets: dict = {}
        super().__init__(params, dict(lr=lr, betas=tuple(betas), eps=eps, weight_decay=weight_decay,
                                      state_bits=state_bits, seed=seed))

    def __setstate__(self, state):
        """Also what load_state_dict, copies and unpickling come through. The
        launches hold addresses, so they are made anew; a saved state of
        groups without a seed takes this optimiser's."""
        super().__setstate__(state)
        self._sets = {}
        self.defaults.setdefault("seed", 0)
        for group in self.param_groups:
            group.setdefault("seed", self.defaults["seed"])

    @property
    def seed(self) -> int:
        return self.param_groups[0]["seed"]

    @seed.setter
    def seed(self, value: int):
        self.defaults["seed"] = value
        for group in self.param_groups:
            group["seed"] = value

    def _new_state(self, p: torch.Tensor, bits: int) -> dict:
        n = p.numel()
        if bits == 32:
            return {"step": 0, "exp_avg": torch.zeros(n, dtype=torch.float32, device=p.device),
                    "exp_avg_sq": torch.zeros(n, dtype=torch.float32, device=p.device)}
        s = {"step": 0}
        for k in ("exp_avg", "exp_avg_sq"):
            s[k] = torch.zeros(n, dtype=torch.uint8, device=p.device).view(torch.float8_e4m3fn)
            s[k + "_scale"] = torch.zeros(-(-n // dpb.STATE_BLOCK), dtype=torch.float32, device=p.device)
        return s

    def _param_sets(self, index: int, group: dict):
        """The group's parameters that have ever had a gradient, by dtype and device, with their states."""
        new = [p for p in group["params"] if p.grad is not None and p not in self.state]
        ids = list(map(id, group["params"]))  # groups and parameters may be taken out or exchanged
        if new or self._sets.get(index, (None,))[0] != ids:
            for p in new:
                if p.is_sparse or p.grad.is_sparse:
                    raise ValueError("AdamW takes dense gradients")
                self.state[p] = self._new_state(p, group["state_bits"])
            kinds: dict = {}
            for p in group["params"]:
                if p in self.state:
                    kinds.setdefault((p.dtype, p.device), []).append(p)
            sets = []
            for ps in kinds.values():
                st = [self.state[p] for p in ps]
                names = ["exp_avg", "exp_avg_sq"] + (["exp_avg_scale", "exp_avg_sq_scale"]
                                                     if group["state_bits"] == 8 else [])
                sets.append((ps, dpb.AdamWGroup(ps, *([s[k] for s in st] for k in names))))
            self._sets[index] = ids, sets
        return self._sets[index][1]

    @torch.no_grad()
    def step(self, closure=None, grad_scale: Optional[torch.Tensor] = None):
        if torch.cuda.is_initialized() and torch.cuda.is_current_stream_capturing():
            raise RuntimeError("AdamW.step() cannot be captured: a replay would repeat this step's bias corrections and bits")
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for index, group in enumerate(self.param_groups):
            for ps, launch in self._param_sets(index, group):
                state, steps = self.state, set()
                for p in ps:
                    if p.grad is not None:
                        state[p]["step"] += 1
                        steps.add(state[p]["step"])
                for n in steps:  # one, unless gradients were missing in earlier steps
                    grads = [None if p.grad is None or state[p]["step"] != n else p.grad.contiguous() for p in ps]
                    launch.step(grads, lr=group["lr"], betas=group["betas"], eps=group["eps"],
                                weight_decay=group["weight_decay"], step=n, seed=group["seed"] + index,
                                grad_scale=grad_scale)
        return loss

    def add_param_group(self, group):
        super().add_param_group(group)
        self._sets.clear()

    def load_state_dict(self, state_dict):
        """As torch's, but the states keep their own dtypes (torch casts them to the parameters')."""
        super().load_state_dict(state_dict)
        ids = [i for g in state_dict["param_groups"] for i in g["params"]]
        ps = [p for g in self.param_groups for p in g["params"]]
        for i, p in zip(ids, ps):
            if i in state_dict["state"]:
                self.state[p] = {k: v.clone().to(p.device) if isinstance(v, torch.Tensor) else v
                                 for k, v in state_dict["state"][i].items()}
        self._sets.clear()
