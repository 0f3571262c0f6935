"""What the orthogonalised updates take at the edges of their contract: lists packed into one buffer, lists that share what is only
read."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _flat(shapes, gen):
    """One buffer with the matrices one behind the other, and its views."""
    sizes = [s[0] * s[1] for s in shapes]
    buffer = torch.randn(sum(sizes), generator=gen).cuda()
    return [t.view(s) for t, s in zip(buffer.split(sizes), shapes)]


def test_packed_lists_and_shared_gradients(lp):
    """Neighbours in one buffer do not overlap, and several lists may read the same gradient."""
    gen = torch.Generator().manual_seed(2)
    shapes = [(8, 8), (64, 64), (100, 90), (20, 300)]
    mats = _flat(shapes, gen)
    want = [lp.orthogonalize([g.clone()])[0] for g in mats[:3]]
    ws = torch.empty(lp.lp_orthogonalize_workspace_bytes(mats), dtype=torch.uint8, device="cuda")
    lp.lp_orthogonalize(mats, mats, ws)   # in place
    assert all(torch.equal(a, b) for a, b in zip(mats, want))
    w, m = _flat([(64, 64)] * 2, gen), [torch.zeros(64, 64, device="cuda") for _ in range(2)]
    w[1].copy_(w[0])
    g = torch.randn(64, 64, generator=gen).cuda()
    lp.muon_step(w, [g, g], m, lr=0.1)
    assert torch.equal(w[0], w[1]) and torch.equal(m[0], m[1]) and torch.equal(m[0], g)
    with pytest.raises(lp.LightplaneError, match="overlap"):
        lp.muon_step([w[0], w[0]], [g, g], m, lr=0.1)


def _reference(g, steps=5):
    x = g.double().cpu()
    x = x / (x.square().sum((-2, -1), keepdim=True).sqrt() + 1e-7)
    for _ in range(steps):
        s = x @ x.mT
        x = 3.4445 * x + (-4.775 * s + 2.0315 * s @ s) @ x
    return x


def test_what_else_a_call_holds(lp):
    """Matrices of at most 64 x 128 come out with the same bits whatever stands beside them; of larger ones the order of sums follows
    the work of the whole call, so they are held to the formula in 64 bits both times (5e-5 of the result's norm: five steps that
    magnify fp32 rounding up to 485 times in directions of small singular values)."""
    gen = torch.Generator().manual_seed(6)
    rand = lambda *s: torch.randn(*s, generator=gen).cuda()  # noqa: E731
    same = [rand(64, 128), rand(128, 64), rand(3, 33, 100), rand(64, 64), rand(1, 128)]
    beside = [rand(300, 100, 100), rand(700, 900), rand(120, 30, 400)]
    for g, o in zip(same, lp.orthogonalize(same + beside)):
        assert torch.equal(o, lp.orthogonalize([g])[0])
    among, alone = lp.orthogonalize(beside)[0][0], lp.orthogonalize([beside[0][0].contiguous()])[0]
    want = _reference(beside[0][0])
    for o in (among, alone):
        assert float((o.double().cpu() - want).norm()) <= 5e-5 * float(want.norm())
