"""The operators of a training step through torch: the norm as an autograd function, Muon as an optimiser, and the example that
runs them with the Splatter and the Renderer."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("occupied", [False, True])
def test_group_norm_gradients_are_the_librarys(lp, occupied):
    from paper_2404_19760_amd import autograd as lpa
    gen = torch.Generator().manual_seed(4)
    x = torch.randn(2, 9, 8, 7, 16, generator=gen).cuda().requires_grad_(True)
    gamma, beta = (torch.randn(16, generator=gen).cuda().requires_grad_(True) for _ in range(2))
    occ = (torch.rand(x.shape[:-1], generator=gen) - 0.4).cuda() if occupied else None
    w = torch.randn(x.shape, generator=gen).cuda()
    y = lpa.group_norm(x, 4, gamma, beta, lp.LP_ACT_SILU, 1e-5, occ)
    (y * w).sum().backward()
    norm = lp.GroupNorm(4, gamma.detach(), beta.detach(), lp.LP_ACT_SILU, 1e-5, occ)
    want, stats = lp.group_norm_fwd(norm, x.detach())
    d_x, d_gamma, d_beta = lp.group_norm_bwd(norm, x.detach(), stats, w)
    assert torch.equal(y, want) and torch.equal(x.grad, d_x) and torch.equal(gamma.grad, d_gamma) and torch.equal(beta.grad, d_beta)


def test_group_norm_gradients_of_some_inputs(lp):
    from paper_2404_19760_amd import autograd as lpa
    x = torch.randn(1, 300, 8, device="cuda")
    gamma = torch.ones(8, device="cuda", requires_grad=True)
    lpa.group_norm(x, 2, gamma, None, lp.LP_ACT_NONE).square().sum().backward()
    # sum of (gamma xh)^2: the gradient of gamma is 2 sum xh^2, 2 x 300 x 4 over a group's four channels (but for eps)
    assert torch.allclose(gamma.grad.view(2, 4).sum(1), torch.full((2,), 2400.0, device="cuda"), rtol=1e-4)
    y = lpa.group_norm(x.requires_grad_(True), 2, dtype=torch.bfloat16)
    assert y.dtype == torch.bfloat16
    y.float().sum().backward()   # (sums over a group do not change)
    assert float(x.grad.abs().max()) < 1e-4


def test_muon_optimiser_steps_the_librarys_way(lp):
    from paper_2404_19760_amd.optim import Muon
    gen = torch.Generator().manual_seed(1)
    params = [torch.randn(s, generator=gen).cuda().requires_grad_(True) for s in ((64, 16), (3, 64, 64), (100, 200))]
    idle = torch.randn(8, 8, device="cuda", requires_grad=True)
    opt = Muon(params + [idle], lr=0.1, momentum=0.9, weight_decay=0.01)
    w, m = [p.detach().clone() for p in params], [torch.zeros_like(p) for p in params]
    kept = idle.detach().clone()
    for step in range(2):
        for p in params:
            p.grad = torch.randn(p.shape, generator=gen).cuda()
        opt.step()
        lp.muon_step(w, [p.grad for p in params], m, lr=0.1, momentum=0.9, weight_decay=0.01)
    assert all(torch.equal(a, b) for a, b in zip(w, params)) and torch.equal(idle, kept)
    state = opt.state_dict()
    assert all(torch.equal(state["state"][k]["momentum"], v) for k, v in enumerate(m))
    with pytest.raises(ValueError):
        Muon([torch.zeros(8, device="cuda")])
    with pytest.raises(ValueError):
        Muon([torch.zeros(8, 8, device="cuda", dtype=torch.float16)])


def test_example_fits_views(lp):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import fit_views
    finally:
        sys.path.pop(0)
    losses = fit_views.fit(steps=40, res=24, size=32, samples=48, n_views=4, log=None)
    assert losses[-1] < 0.5 * losses[0], losses
