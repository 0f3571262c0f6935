"""torch.autograd wrappers, for callers that train with PyTorch optimisers.  Argument marshalling only: every step runs in the
library's kernels.

render: the Renderer's two entry points; the forward keeps one scalar per ray (Section 3.4: the backward recomputes the
rest), the backward calls lp_render_bwd.  No gradient flows to the rays (the library produces none); first derivatives alone.
group_norm: group norm with an activation over channel-last grids; the forward keeps its input, the occupancy and two
numbers a group; first derivatives alone.
linear: a product with bias, activation and residual; keeps its input, the weight and, where there is an activation, what goes into it.
residual_norm: the norms around a residual block; keeps its inputs, the backward computes the rest again."""
from typing import List, Optional, Sequence

import torch

from . import (LP_ACT_NONE, LP_MATH_DEFAULT, LP_NORM_RMS, Grid, GroupNorm, Linear, Mlp, Rays, ResidualNorm, group_norm_fwd, linear_fwd,
               lp_bwd_workspace_bytes, lp_group_norm_bwd, lp_group_norm_workspace_bytes, lp_linear_bwd, lp_linear_workspace_bytes,
               lp_render_bwd, lp_render_fwd, lp_residual_norm_bwd, lp_residual_norm_workspace_bytes, residual_norm_fwd)


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


def _like(t: torch.Tensor) -> torch.Tensor:
    return torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device=t.device)


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, act, x, weight, bias, residual):
        w = weight.detach().to(x.dtype)
        detach = lambda t: None if t is None else t.detach()
        keep = act != LP_ACT_NONE and any(ctx.needs_input_grad[1:4])
        y, pre = linear_fwd(Linear(w, detach(bias), act), x.detach(), detach(residual), keep)
        # (a weight that was cast is kept as it was used; the parameter itself is kept for its version and for second derivatives)
        ctx.save_for_backward(x, weight, bias, pre, None if w.dtype == weight.dtype else w)
        ctx.lp = act
        return y

    @staticmethod
    def backward(ctx, upstream):
        x, weight, bias, pre, w = ctx.saved_tensors
        need_x, need_weight, need_bias, need_residual = ctx.needs_input_grad[1:5]
        linear = Linear(weight.detach() if w is None else w, None if bias is None else bias.detach(), ctx.lp)
        d_y = upstream.contiguous()
        d_x = _like(x) if need_x else None
        d_weight = torch.zeros(weight.shape, dtype=torch.float32, device=x.device) if need_weight else None
        d_bias = torch.zeros_like(bias) if need_bias else None
        if need_x or need_weight or need_bias:
            ws = torch.empty(lp_linear_workspace_bytes(linear, x.detach())[1], dtype=torch.uint8, device=x.device)
            lp_linear_bwd(linear, x.detach(), pre, d_y, d_x, d_weight, d_bias, ws)
        if d_weight is not None:
            d_weight = d_weight.to(weight.dtype)
        d_x, d_weight, d_bias = _first((d_x, d_weight, d_bias), (upstream, x, weight, bias))
        return None, d_x, d_weight, d_bias, upstream if need_residual else None


def linear(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, act: int = LP_ACT_NONE,
           residual: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Differentiable act(x W^T + b) + residual (see Linear); gradients flow to x, weight, bias and residual.  A weight of another
    type (fp32, as the optimisers have it) is rounded to that of x; its gradient is summed in fp32."""
    return _Linear.apply(int(act), x, weight, bias, residual)


class _ResidualNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, spec, h, f, gamma, beta, post_gamma, gate):
        kind, post_norm, alpha, eps, dtype = spec
        detach = lambda t: None if t is None else t.detach()
        norm = ResidualNorm(kind, detach(gamma), detach(beta), post_norm, detach(post_gamma), detach(gate), alpha, eps)
        s, y = residual_norm_fwd(norm, h.detach(), detach(f), dtype)
        ctx.save_for_backward(h, f, gamma, beta, post_gamma, gate)
        ctx.lp = spec
        ctx.set_materialize_grads(False)
        return h if f is None and alpha == 1.0 else s, y   # (residual_norm_fwd: without a block s is h itself)

    @staticmethod
    def backward(ctx, up_s, up_y):
        kind, post_norm, alpha, eps, _ = ctx.lp
        h, f, gamma, beta, post_gamma, gate = ctx.saved_tensors
        if up_s is None and up_y is None:
            return (None,) * 7
        norm = ResidualNorm(kind, gamma, beta, post_norm, post_gamma, gate, alpha, eps)
        d_s = up_s if up_s is None or up_s.stride() == h.stride() else _like(h).copy_(up_s)
        d_y = None if up_y is None else up_y.contiguous()
        needs = ctx.needs_input_grad[1:]
        d_h = _like(h) if needs[0] else None
        d_f = _like(f) if needs[1] else None
        params = [torch.zeros_like(p) if need else None for p, need in zip((gamma, beta, post_gamma, gate), needs[2:])]
        with_f = params if f is not None else [*params[:2], None, None]
        ws = torch.empty(lp_residual_norm_workspace_bytes(norm, h), dtype=torch.uint8, device=h.device)
        lp_residual_norm_bwd(norm, h, f, d_s, d_y, d_h, d_f, *with_f, ws)
        return (None, *_first((d_h, d_f, *params), (up_s, up_y, h, f, gamma, beta, post_gamma, gate)))


def residual_norm(h: torch.Tensor, f: Optional[torch.Tensor] = None, gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None,
                  kind: int = LP_NORM_RMS, post_norm: bool = False, post_gamma: Optional[torch.Tensor] = None,
                  gate: Optional[torch.Tensor] = None, alpha: float = 1.0, eps: float = 1e-5, dtype=None):
    """Differentiable norms around a residual block (see ResidualNorm): (s, y) for the sum h so far and the block's result f, or None
    (then dtype: of y); gradients flow to h, f, gamma, beta, post_gamma and gate."""
    return _ResidualNorm.apply((int(kind), bool(post_norm), float(alpha), float(eps), dtype), h, f, gamma, beta, post_gamma, gate)
