"""A torch.optim optimiser on the library's orthogonalised update (lp_muon_step), for the weight matrices of decoders and of networks
around them.  Vectors (biases, norm parameters) and structures belong to another optimiser.  And what stands before the optimisers'
steps: the gradients of all parameters brought under a largest norm (lp_clip_grad_norm)."""
from typing import Iterable, Union

import torch

from . import LP_MUON_SCALE_ASPECT, clip_grad_norm, muon_step


class Muon(torch.optim.Optimizer):
    """params: float32 GPU tensors [...][rows][cols], contiguous; leading axes count matrices (the decoders of several scenes).
    All matrices of a parameter group are stepped in one call."""

    def __init__(self, params: Iterable, lr: float = 0.02, momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0,
                 scale: int = LP_MUON_SCALE_ASPECT, steps: int = 5, coeffs=None, eps: float = 1e-7):
        super().__init__(params, dict(lr=lr, momentum=momentum, nesterov=nesterov, weight_decay=weight_decay, scale=scale,
                                      steps=steps, coeffs=coeffs, eps=eps))

    def add_param_group(self, param_group):
        super().add_param_group(param_group)
        if any(p.dim() < 2 or p.dtype != torch.float32 for p in self.param_groups[-1]["params"]):
            self.param_groups.pop()
            raise ValueError("Muon takes float32 matrices [...][rows][cols]")

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for group in self.param_groups:
            params = [p for p in group["params"] if p.grad is not None]
            for p in params:
                if "momentum" not in self.state[p]:
                    self.state[p]["momentum"] = torch.zeros_like(p, memory_format=torch.contiguous_format)
            muon_step([p.detach() for p in params], [p.grad.contiguous() for p in params], [self.state[p]["momentum"] for p in params],
                      lr=group["lr"], momentum=group["momentum"], nesterov=group["nesterov"], weight_decay=group["weight_decay"],
                      scale=group["scale"], steps=group["steps"], coeffs=group["coeffs"], eps=group["eps"])
        return loss


@torch.no_grad()
def clip_grad_norm_(params: Union[torch.Tensor, Iterable[torch.Tensor]], max_norm: float, eps: float = 1e-6) -> torch.Tensor:
    """Scales the gradients of all parameters, in place, by min(1, max_norm / (norm + eps)), and returns the norm of all of them
    together before that, on the GPU (nothing waits for it).  Parameters without a gradient do not take part; gradients are dense GPU
    tensors.  A norm that is not finite is applied as it is."""
    params = [params] if isinstance(params, torch.Tensor) else list(params)
    grads, seen = [], set()
    for p in params:
        if p.grad is not None and id(p.grad) not in seen:   # (a parameter listed twice has one gradient)
            seen.add(id(p.grad))
            grads.append(p.grad)
    if not grads:
        return torch.zeros((), device=params[0].device if params else None)
    return clip_grad_norm(grads, max_norm, eps)
