"""A torch.optim optimiser on the library's orthogonalised update (lp_muon_step), for the weight matrices of decoders and of networks
around them.  Vectors (biases, norm parameters) and structures belong to another optimiser."""
from typing import Iterable

import torch

from . import LP_MUON_SCALE_ASPECT, muon_step


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
