"""An optimizer whose update of a matrix is its momentum, orthogonalised: every direction that the gradients of a matrix point in is
followed at about the same rate, strong and weak ones alike.

Matrices go through ``binding.fsa_orthogonalize`` (those of one size and type in one call); whatever is no matrix has to go
to another optimizer.
"""
from __future__ import annotations

from typing import Iterable

import torch

from . import binding


class OrthogonalMomentum(torch.optim.Optimizer):
    """m = momentum * m + grad;  p -= rate * (decay * p + sqrt(max(1, rows / columns)) * orthogonalised(m)), or, with `nesterov`, of
    grad + momentum * m.  The momentum is fp32 whatever the matrix's type, and so is the step, of which a 16-bit matrix is rounded once."""

    def __init__(self, params: Iterable, rate: float = 0.02, momentum: float = 0.95, *, nesterov: bool = True, decay: float = 0.0,
                 steps: int = 5, coefficients=binding.ORTHOGONAL_COEFFICIENTS, eps: float = 1e-7):
        if rate < 0.0 or not 0.0 <= momentum < 1.0 or decay < 0.0:
            raise ValueError("rate and decay must not be negative, momentum must be in [0, 1)")
        super().__init__(params, dict(rate=rate, momentum=momentum, nesterov=nesterov, decay=decay, steps=steps,
                                      coefficients=coefficients, eps=eps))

    def add_param_group(self, param_group):
        super().add_param_group(param_group)
        for p in self.param_groups[-1]["params"]:
            if p.dim() != 2:
                self.param_groups.pop()
                raise ValueError("only matrices have an orthogonalised update, got %s" % (tuple(p.shape),))

    def load_state_dict(self, state_dict):
        super().load_state_dict(state_dict)
        # torch brings what is loaded to the parameters' type: the momentum stays fp32
        names = [i for group in state_dict["param_groups"] for i in group["params"]]
        for i, p in zip(names, (p for group in self.param_groups for p in group["params"])):
            if "momentum" in state_dict["state"].get(i, ()):
                self.state[p]["momentum"] = state_dict["state"][i]["momentum"].detach().to(p.device, torch.float32, copy=True)

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for group in self.param_groups:
            alike = {}
            for p in group["params"]:
                if p.grad is None or p.numel() == 0:
                    continue
                state = self.state[p]
                grad = p.grad.float()
                if "momentum" not in state:
                    state["momentum"] = torch.zeros_like(grad, memory_format=torch.contiguous_format)
                m = state["momentum"].mul_(group["momentum"]).add_(grad)
                alike.setdefault((tuple(p.shape), p.device), []).append((p, grad.add(m, alpha=group["momentum"]) if group["nesterov"] else m))
            for (shape, _), members in alike.items():
                # (a lone one lies as its gradient does, whose columns may be what is contiguous)
                update = members[0][1].contiguous()[None] if len(members) == 1 else torch.stack([u for _, u in members])
                update = binding.fsa_orthogonalize(update, group["coefficients"], group["steps"], eps=group["eps"],
                                                   scale=max(1.0, shape[0] / shape[1]) ** 0.5)
                for (p, _), u in zip(members, update):
                    # 16-bit parameters are rounded once: a decay by itself, mostly less than half of a step, would be rounded away
                    wide = p.float() if p.dtype in (torch.bfloat16, torch.float16) else p
                    if group["decay"]:
                        wide.mul_(1.0 - group["rate"] * group["decay"])
                    wide.add_(u, alpha=-group["rate"])
                    if wide is not p:
                        p.copy_(wide)
        return loss
