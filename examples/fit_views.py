"""Lifts views of a scene into a voxel grid and trains a small network on it, from the Splatter to the optimiser:

    pixel features -> Splatter -> grid (+ a learned one) -> group norm + SiLU over the cells the Splatter reached
        -> residual block over the cells (layer norm, product + SiLU, product + residual) -> Renderer -> loss

Gradients are clipped by their norm; the matrices of the decoder and of the block are stepped by Muon (orthogonalised updates), everything
else by Adam.  The views are rendered from a random
scene by the library itself.  Needs a GPU:

    python examples/fit_views.py [--steps 200] [--res 48] [--size 64]
"""
import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2404_19760_amd as lp  # noqa: E402
from paper_2404_19760_amd import autograd as lp_autograd  # noqa: E402
from paper_2404_19760_amd.optim import Muon, clip_grad_norm_  # noqa: E402

CHANNELS, HIDDEN, GROUPS = 16, 64, 4
BG = (1.0, 1.0, 1.0)


def views(count, size, samples, gen):
    """Rays of `count` square images from cameras around the origin."""
    at = torch.randn(count, 3, generator=gen, device="cuda")
    at = 2.5 * at / at.norm(dim=1, keepdim=True)
    forward = -at / at.norm(dim=1, keepdim=True)
    right = torch.linalg.cross(forward, torch.tensor([0.0, 0.0, 1.0], device="cuda").expand_as(forward))
    right = right / right.norm(dim=1, keepdim=True)
    up = torch.linalg.cross(right, forward)
    u = (torch.arange(size, device="cuda") + 0.5) / size * 2 - 1
    v, u = torch.meshgrid(u, u, indexing="ij")
    d = forward[:, None, None] + 0.5 * (u[None, ..., None] * right[:, None, None] - v[None, ..., None] * up[:, None, None])
    d = (d / d.norm(dim=-1, keepdim=True)).reshape(-1, 3).contiguous()
    m = d.shape[0]
    origins = at[:, None].expand(count, size * size, 3).reshape(-1, 3).contiguous()
    return lp.Rays(origins, d, torch.full((m,), 1.0, device="cuda"), torch.full((m,), 4.0, device="cuda"), samples)


def mlp(gen):
    dims = (CHANNELS, HIDDEN, HIDDEN, 4)
    w = [torch.randn(o, i, generator=gen, device="cuda") * (2.0 / i) ** 0.5 for i, o in zip(dims, dims[1:])]
    return lp.Mlp(w, [torch.zeros(o, device="cuda") for o in dims[1:]])


def fit(steps=200, res=48, size=64, samples=64, n_views=8, seed=0, log=print):
    """Returns the losses."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    shape = (res, res, res)
    # the scene: a smooth random grid, denser in the middle
    coarse = torch.randn(1, CHANNELS, 6, 6, 6, generator=gen, device="cuda")
    scene = 2 * torch.nn.functional.interpolate(coarse, size=shape, mode="trilinear", align_corners=True).permute(0, 2, 3, 4, 1).contiguous()
    rays = views(n_views, size, samples, gen)
    target, _, _, _ = lp.render_fwd(lp.Grid(lp.LP_GRID_VOXEL, [scene], shape), mlp(gen), rays, BG)
    # pixel features: a fixed projection of the colours, pushed along the rays
    feats = (target - 0.5) @ torch.randn(3, CHANNELS, generator=gen, device="cuda")
    grid = lp.target_struct(lp.LP_GRID_VOXEL, 1, CHANNELS, shape)
    (lifted,), (weight,) = lp.splat_fwd(grid, rays, lp.Splat(feats.contiguous()))

    net = mlp(gen)
    latent = torch.zeros_like(lifted, requires_grad=True)
    gamma, beta = (torch.full((CHANNELS,), v, device="cuda", requires_grad=True) for v in (1.0, 0.0))
    # the block: its last matrix is zero, so that it starts as nothing beside the sum
    block = [torch.randn(2 * CHANNELS, CHANNELS, generator=gen, device="cuda") * (2.0 / CHANNELS) ** 0.5, torch.zeros(CHANNELS, 2 * CHANNELS, device="cuda")]
    block_biases = [torch.zeros(2 * CHANNELS, device="cuda"), torch.zeros(CHANNELS, device="cuda")]
    for t in net.weights + net.biases + block + block_biases:
        t.requires_grad_(True)
    muon = Muon(net.weights + block, lr=0.02)
    adam = torch.optim.Adam([latent, gamma, beta, *net.biases, *block_biases], lr=2e-2)
    params = [p for o in (muon, adam) for g in o.param_groups for p in g["params"]]
    losses = []
    for step in range(steps):
        x = lp_autograd.group_norm(lifted + latent, GROUPS, gamma, beta, lp.LP_ACT_SILU, occupancy=weight)
        h, normed = lp_autograd.residual_norm(x, kind=lp.LP_NORM_LAYER)
        x = lp_autograd.linear(lp_autograd.linear(normed, block[0], block_biases[0], lp.LP_ACT_SILU), block[1], block_biases[1], residual=h)
        rgb, _, _ = lp_autograd.render(lp.Grid(lp.LP_GRID_VOXEL, [x], shape), net, rays, BG)
        loss = (rgb - target).square().mean()
        muon.zero_grad()
        adam.zero_grad()
        loss.backward()
        clip_grad_norm_(params, 1.0)
        muon.step()
        adam.step()
        losses.append(loss.detach())
        if log and (step % 20 == 0 or step + 1 == steps):
            log(f"step {step:4d}  loss {float(losses[-1]):.5f}", flush=True)
    return [float(v) for v in losses]


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--res", type=int, default=48)
    ap.add_argument("--size", type=int, default=64)
    a = ap.parse_args()
    fit(a.steps, a.res, a.size)
