"""torch.autograd wrappers, for callers that train with PyTorch optimisers.  Argument marshalling only: every step runs in the
library's kernels.

render: the Renderer's two entry points; the forward keeps one scalar per ray (Section 3.4: the backward recomputes the
rest), the backward calls lp_render_bwd.  No gradient flows to the rays (the library produces none); first derivatives alone.
group_norm: group norm with an activation over channel-last grids; the forward keeps its input, the occupancy and two
numbers a group; first derivatives alone."""
from typing import List, Optional, Sequence

import torch

from . import (LP_ACT_NONE, LP_MATH_DEFAULT, Grid, GroupNorm, Mlp, Rays, group_norm_fwd, lp_bwd_workspace_bytes,
               lp_group_norm_bwd, lp_group_norm_workspace_bytes, lp_render_bwd, lp_render_fwd)


class _First(torch.autograd.Function):
    """Results of a backward that is not differentiable itself, where a graph of it is asked for (create_graph): derivatives of
    them are an error.  (torch's once_differentiable sees to that only where the upstream gradient has a graph; a gradient
    penalty's has none, its second derivatives come from the inputs.)"""
    @staticmethod
    def forward(ctx, count, *tensors):
        return tuple(t.view_as(t) for t in tensors[:count])

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("the library's operators have first derivatives alone")


def _first(results, inputs):
    """`results` (None: not wanted), which depend on `inputs` in a way that no graph holds."""
    if not torch.is_grad_enabled():
        return results
    there = [t for t in results if t is not None]
    marked = iter(_First.apply(len(there), *there, *[t for t in inputs if t is not None]) if there else ())
    return tuple(None if t is None else next(marked) for t in results)


class _Render(torch.autograd.Function):
    @staticmethod
    def forward(ctx, spec, n_grid: int, n_layers: int, *tensors):
        kind, res, aabb_min, aabb_max, contract_a, t_range, rays, bg, math_mode = spec
        data = [t.detach() for t in tensors[:n_grid]]
        weights = [t.detach() for t in tensors[n_grid:n_grid + n_layers]]
        biases = [t.detach() for t in tensors[n_grid + n_layers:]]
        grid = Grid(kind=kind, data=data, res=res, aabb_min=aabb_min, aabb_max=aabb_max, contract_a=contract_a,
                    t_range=t_range)
        mlp = Mlp(weights=weights, biases=biases)
        m, dev = rays.n_rays, rays.origins.device
        rgb = torch.empty((m, 3), dtype=torch.float32, device=dev)
        alpha = torch.empty((m,), dtype=torch.float32, device=dev)
        depth = torch.empty((m,), dtype=torch.float32, device=dev)
        cache = torch.empty((m,), dtype=torch.float32, device=dev)
        lp_render_fwd(grid, mlp, rays, bg, rgb, alpha, depth, cache, math_mode)
        ctx.lp = (grid, mlp, rays, bg, math_mode, cache)
        ctx.inputs = tensors
        ctx.mark_non_differentiable(cache)
        return rgb, alpha, depth

    @staticmethod
    def backward(ctx, d_rgb, d_alpha, d_depth):
        grid, mlp, rays, bg, math_mode, cache = ctx.lp
        dev = rays.origins.device
        d_grid = [torch.zeros_like(t, dtype=torch.float32) for t in grid.data]
        dW = [torch.zeros_like(w) for w in mlp.weights]
        db = [torch.zeros_like(b) for b in mlp.biases]
        ws = torch.empty(lp_bwd_workspace_bytes(grid, mlp, rays, math_mode), dtype=torch.uint8, device=dev)
        as_f32 = lambda t: None if t is None else t.contiguous().float()
        lp_render_bwd(grid, mlp, rays, bg, as_f32(d_rgb), as_f32(d_alpha), as_f32(d_depth), cache, d_grid, dW, db, ws,
                      math_mode)
        # gradients of structures stored in reduced precision come back in that type
        d_grid = [g.to(t.dtype) for g, t in zip(d_grid, grid.data)]
        return (None, None, None, *_first((*d_grid, *dW, *db), (d_rgb, d_alpha, d_depth, *ctx.inputs)))


def render(grid: Grid, mlp: Mlp, rays: Rays, bg: Sequence[float], math_mode: int = LP_MATH_DEFAULT):
    """Differentiable Renderer: returns (rgb [M][3], alpha [M], depth [M]); gradients flow to
    grid.data, mlp.weights and mlp.biases (tensors with requires_grad)."""
    spec = (grid.kind, tuple(grid.res), tuple(grid.aabb_min), tuple(grid.aabb_max), float(grid.contract_a),
            tuple(grid.t_range), rays, tuple(float(v) for v in bg), int(math_mode))
    return _Render.apply(spec, len(grid.data), len(mlp.weights), *grid.data, *mlp.weights, *mlp.biases)


class _GroupNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, spec, x, gamma, beta, occupancy):
        groups, act, eps, dtype = spec
        detach = lambda t: None if t is None else t.detach()
        norm = GroupNorm(groups, detach(gamma), detach(beta), act, eps, occupancy)
        y, stats = group_norm_fwd(norm, x.detach(), dtype)
        ctx.save_for_backward(x, gamma, beta, occupancy, stats)
        ctx.lp = spec
        return y

    @staticmethod
    def backward(ctx, upstream):
        groups, act, eps, _ = ctx.lp
        x, gamma, beta, occupancy, stats = ctx.saved_tensors
        norm = GroupNorm(groups, gamma, beta, act, eps, occupancy)
        need_x, need_gamma, need_beta = ctx.needs_input_grad[1:4]
        d_y = upstream.contiguous()
        d_x = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=x.device) if need_x else None
        d_gamma = torch.zeros_like(gamma) if need_gamma else None
        d_beta = torch.zeros_like(beta) if need_beta else None
        n = lp_group_norm_workspace_bytes(norm, x, d_y.dtype)[1]
        ws = torch.empty(n, dtype=torch.uint8, device=x.device) if n else None
        lp_group_norm_bwd(norm, x, stats, d_y, d_x, d_gamma, d_beta, ws)
        d_x, d_gamma, d_beta = _first((d_x, d_gamma, d_beta), (upstream, x, gamma, beta))
        return None, d_x, d_gamma, d_beta, None


def group_norm(x: torch.Tensor, groups: int, gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None,
               act: int = LP_ACT_NONE, eps: float = 1e-5, occupancy: Optional[torch.Tensor] = None, dtype=None) -> torch.Tensor:
    """Differentiable group norm with an activation of a channel-last tensor [N][...][C] (see GroupNorm; dtype: of the result);
    gradients flow to x, gamma and beta."""
    return _GroupNorm.apply((int(groups), int(act), float(eps), dtype), x, gamma, beta, occupancy)
