"""Lifts views of a scene into a voxel grid and trains a small network on it, from the Splatter to the optimiser:

    pixel features -> Splatter -> grid (+ a learned one) -> group norm + SiLU over the cells the Splatter reached -> Renderer -> loss

The decoder's matrices are stepped by Muon (orthogonalised updates), everything else by Adam.  The views are rendered from a random
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
from paper_2404_19760_amd.optim import Muon  # noqa: E402

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
    for t in net.weights + net.biases:
        t.requires_grad_(True)
    muon = Muon(net.weights, lr=0.02)
    adam = torch.optim.Adam([latent, gamma, beta, *net.biases], lr=2e-2)
    losses = []
    for step in range(steps):
        x = lp_autograd.group_norm(lifted + latent, GROUPS, gamma, beta, lp.LP_ACT_SILU, occupancy=weight)
        rgb, _, _ = lp_autograd.render(lp.Grid(lp.LP_GRID_VOXEL, [x], shape), net, rays, BG)
        loss = (rgb - target).square().mean()
        muon.zero_grad()
        adam.zero_grad()
        loss.backward()
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
