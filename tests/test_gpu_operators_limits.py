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
