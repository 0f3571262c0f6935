"""Orthogonalisation by Newton-Schulz products and the optimiser step on it, against the formulas in 64 bits.

Tolerances: five steps magnify an error in a direction of small singular value up to 3.4445^5 = 485 times.  Operands of 22 bits
and sums in fp32 put 2^-22 of X's size into X in every step, of which such directions hold their share: for gradients of a few
strong directions above noise, as here, some 1e-5 of the result's norm is reached; 5e-5 is allowed (2-norm over 2-norm), 16-bit results add their own
rounding (2^-9, 2^-12 in the mean).  A largest difference is held to 40 times that of the results' root mean square."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

COEFFS = (3.4445, -4.775, 2.0315)
TOL = {torch.float32: 5e-5, torch.bfloat16: 3e-3, torch.float16: 4e-4}


def reference(g, steps=5, coeffs=COEFFS, eps=1e-7):
    x = g.double().cpu()
    norm = x.square().sum((-2, -1), keepdim=True).sqrt()
    x = torch.where(norm > 0, x / (norm + eps), x)
    tall = x.shape[-2] > x.shape[-1]
    x = x.mT.contiguous() if tall else x
    per_step = [coeffs] * steps if isinstance(coeffs[0], float) else coeffs
    for a, b, c in per_step:
        s = x @ x.mT
        x = a * x + (b * s + c * s @ s) @ x
    return x.mT if tall else x


def gradient(shape, seed, scale=1.0, noise=0.1):
    gen = torch.Generator().manual_seed(seed)
    rank = max(1, min(shape[-2:]) // 6)
    g = torch.randn(*shape[:-1], rank, generator=gen) @ torch.randn(*shape[:-2], rank, shape[-1], generator=gen) / math.sqrt(rank)
    return (scale * (g + noise * torch.randn(shape, generator=gen))).cuda()


def _close(got, want, dtype, label):
    got = got.double().cpu()
    assert torch.isfinite(got).all(), label
    d, norm = got - want, float(want.norm())
    assert float(d.norm()) <= TOL[dtype] * norm, f"{label}: {float(d.norm()) / norm}"
    rms = norm / math.sqrt(want.numel())
    assert float((d.abs() / want.abs().clamp(min=rms)).max()) <= 40 * TOL[dtype], label


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", [(1, 1), (1, 7), (5, 1), (4, 64), (64, 16), (64, 64), (63, 65), (3, 20, 31), (2, 64, 123), (2, 64, 700),
                                   (65, 64), (128, 128), (2, 97, 129), (300, 40), (130, 517), (517, 200), (256, 256), (3, 2, 33, 31)])
def test_against_64_bits(lp, dtype, shape):
    g = gradient(shape, sum(shape)).to(dtype)
    out, = lp.orthogonalize([g])
    assert out.dtype == dtype and out.shape == g.shape
    _close(out, reference(g), dtype, str(shape))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", [(64, 224), (64, 193), (33, 192), (40, 129), (224, 64), (30, 448), (448, 32), (5, 300), (390, 17),
                                   (3, 20, 260), (2, 200, 61), (1, 448), (64, 225), (32, 449), (33, 225)])
def test_long_matrices_of_one_workgroup(lp, dtype, shape):
    """Few rows and up to 224 or 448 columns, and the first ones that are too long."""
    g = gradient(shape, sum(shape)).to(dtype)
    out, = lp.orthogonalize([g])
    _close(out, reference(g), dtype, str(shape))


def test_steps_of_long_and_short_weights(lp):
    """The optimiser over lists of every kind of kernel, in one call."""
    shapes = [(64, 224), (2, 448, 30), (64, 64), (100, 100), (7, 300)]
    gen = torch.Generator().manual_seed(8)
    w = [torch.randn(s, generator=gen).cuda() for s in shapes]
    m = [0.1 * torch.randn(s, generator=gen).cuda() for s in shapes]
    g = [gradient(s, 70 + k) for k, s in enumerate(shapes)]
    before = [(a.clone(), b.clone()) for a, b in zip(w, m)]
    lp.muon_step(w, g, m, lr=0.1, momentum=0.8, weight_decay=0.05)
    for (w0, m0), w1, g1, m1 in zip(before, w, g, m):
        rw, rm = _muon_reference(w0, g1, m0, 0.1, 0.8, True, 0.05, 1)
        assert torch.allclose(m1.double().cpu(), rm, rtol=1e-6, atol=1e-7)
        assert float((w1.double().cpu() - rw).norm()) <= 5e-5 * float((rw - w0.double().cpu()).norm()) + 1e-7 * float(rw.norm())


@pytest.mark.parametrize("count", [1, 120])
def test_long_matrices_beside_large_ones(lp, count):
    """Few of them go with the large ones, many by themselves."""
    mats = [gradient((count, 30, 400), 1), gradient((200, 64), 2), gradient((300, 310), 3), gradient((64, 64), 4)]
    for g, o in zip(mats, lp.orthogonalize(mats)):
        _close(o, reference(g), torch.float32, str(g.shape))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape", [(64, 2999), (100, 5001), (4001, 70), (2, 130, 2500), (300, 1400), (1500, 260)])
def test_long_sums_that_are_divided(lp, dtype, shape):
    """A = X X^T of more than 32 blocks of 32 columns: parts, and their join."""
    g = gradient(shape, sum(shape)).to(dtype)
    out, = lp.orthogonalize([g])
    _close(out, reference(g), dtype, str(shape))


@pytest.mark.parametrize("shapes", [[(100, 200, 300)],                         # 300 tiles of 128 for A, 600 for B X
                                    [(200, 300, 200)],                         # 600 and 1200, tall
                                    [(90, 130, 250), (40, 256, 129), (3, 1, 900)],   # edges in the middle of a tile of 128
                                    [(5, 900, 1000), (700, 700)]])
def test_large_tiles(lp, shapes):
    mats = [gradient(s, 9 + k) for k, s in enumerate(shapes)]
    for g, out in zip(mats, lp.orthogonalize(mats)):
        want = reference(g)
        _close(out, want, torch.float32, str(g.shape))
        if g.dim() == 3:   # the matrices one by one, too
            for i in range(g.shape[0]):
                assert float((out[i].double().cpu() - want[i]).norm()) <= 2 * TOL[torch.float32] * float(want[i].norm()), (g.shape, i)


@pytest.mark.parametrize("shape,dtype", [((262200, 64, 128), torch.bfloat16), ((300, 64, 65536), torch.float32)])
def test_offsets_beyond_32_bits(lp, shape, dtype):
    """Lists of more than 2^31 values and 2^32 bytes: the last matrix is as by itself, zeros stay zeros."""
    mats = torch.zeros(shape, dtype=dtype, device="cuda")
    last = gradient(shape[1:], 3).to(dtype)
    mats[0], mats[-1] = last, last
    alone, = lp.orthogonalize([last], steps=1)
    ws = torch.empty(lp.lp_orthogonalize_workspace_bytes([mats]), dtype=torch.uint8, device="cuda")
    lp.lp_orthogonalize([mats], [mats], ws, steps=1)
    _close(mats[-1], alone.double().cpu(), dtype, "last")
    assert torch.equal(mats[0], mats[-1]) and float(mats[1:-1].abs().amax()) == 0


def test_one_call_for_many_lists(lp):
    """More lists than one set of launches takes, of all sizes and types: each as by itself."""
    shapes = [(64, 16), (64, 64), (4, 64), (2, 100, 30), (7, 300), (129, 65)] * 4
    types = [torch.float32, torch.bfloat16, torch.float16, torch.float32, torch.float32]
    mats = [gradient(s, 50 + k).to(types[k % 5]) for k, s in enumerate(shapes)]
    outs = lp.orthogonalize(mats)
    for g, o in zip(mats, outs):
        single, = lp.orthogonalize([g])
        if g.shape != (7, 300):   # (by itself it is one workgroup's; the reference is what both are held to)
            assert torch.equal(o, single)
        _close(o, reference(g), g.dtype, str(g.shape))
        _close(single, reference(g), g.dtype, str(g.shape))


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e15, 1e37])
def test_scales(lp, scale):
    g = gradient((40, 70), 3) / 10 * scale
    out, = lp.orthogonalize([g], eps=0.0)
    _close(out, reference(g, eps=0.0), torch.float32, str(scale))


@pytest.mark.parametrize("shape", [(30, 40), (200, 90)])
def test_spectra(lp, shape):
    """One strong direction above all others, all directions alike, one entry alone, zeros, NaN in one matrix of several."""
    gen = torch.Generator().manual_seed(5)
    one = torch.randn(shape[0], 1, generator=gen) @ torch.randn(1, shape[1], generator=gen) + 1e-2 * torch.randn(shape, generator=gen)
    same = torch.linalg.qr(torch.randn(max(shape), min(shape), generator=gen))[0]
    same = same if shape[0] > shape[1] else same.mT.contiguous()
    entry = torch.zeros(shape)
    entry[3, 4] = -2.0
    g = torch.stack([one, same, entry, torch.zeros(shape), torch.full(shape, 0.25)]).cuda()
    out, = lp.orthogonalize([g])
    assert float(out[3].abs().max()) == 0
    for k in (0, 1, 2, 4):
        _close(out[k], reference(g[k]), torch.float32, str(k))
    bad = g.clone()
    bad[1, 0, 0] = float("nan")
    bad[2, 0, 0] = float("inf")
    out2, = lp.orthogonalize([bad])
    assert torch.isnan(out2[1]).all() and torch.isnan(out2[2]).any()
    assert torch.equal(out2[0], out[0]) and torch.equal(out2[3:], out[3:])


@pytest.mark.parametrize("shape", [(48, 60), (200, 100)])
@pytest.mark.parametrize("steps,coeffs", [(1, None), (2, None), (9, (1.875, -1.25, 0.375)), (3, (1.5, -0.5, 0.0)),
                                         (3, [(4.0, -6.0, 2.5), (3.0, -3.2, 1.2), (1.875, -1.25, 0.375)])])
def test_coefficients(lp, shape, steps, coeffs):
    g = gradient(shape, 17)
    out, = lp.orthogonalize([g], steps=steps, coeffs=coeffs)
    _close(out, reference(g, steps, coeffs or COEFFS), torch.float32, f"{steps} {coeffs}")


def test_result_is_nearly_orthogonal(lp):
    """With coefficients that converge, rows of the result are orthonormal."""
    g = torch.randn(50, 200, generator=torch.Generator().manual_seed(1)).cuda()
    out, = lp.orthogonalize([g], steps=16, coeffs=(1.875, -1.25, 0.375))
    assert float((out @ out.mT - torch.eye(50, device="cuda")).abs().max()) <= 1e-4


def _muon_reference(w, g, m, lr, mu, nesterov, decay, scale):
    w, g, m = w.double().cpu(), g.double().cpu(), m.double().cpu()
    m = mu * m + g
    o = reference(g + mu * m if nesterov else m)
    r, c = w.shape[-2:]
    s = {0: 1.0, 1: math.sqrt(max(1.0, r / c)), 2: 0.2 * math.sqrt(max(r, c))}[scale]
    return (1 - lr * decay) * w - lr * s * o, m


@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("scale", [0, 1, 2])
def test_muon_step(lp, nesterov, scale):
    shapes = [(64, 16), (4, 64), (3, 64, 64), (200, 70), (70, 300), (2, 40, 500)]
    gen = torch.Generator().manual_seed(3)
    w = [(torch.randn(s, generator=gen) / math.sqrt(s[-1])).cuda() for s in shapes]
    m = [torch.zeros(s, device="cuda") for s in shapes]
    for step in range(3):
        g = [gradient(s, 100 + step, 1e-3) for s in shapes]
        before = [(a.clone(), b.clone()) for a, b in zip(w, m)]
        lp.muon_step(w, g, m, lr=0.05, momentum=0.9, nesterov=nesterov, weight_decay=0.1, scale=scale)
        for (w0, m0), w1, g1, m1 in zip(before, w, g, m):
            rw, rm = _muon_reference(w0, g1, m0, 0.05, 0.9, nesterov, 0.1, scale)
            assert torch.allclose(m1.double().cpu(), rm, rtol=1e-6, atol=1e-9)
            moved = (rw - w0.double().cpu()).norm()
            assert float((w1.double().cpu() - rw).norm()) <= 5e-5 * float(moved) + 1e-7 * float(rw.norm())


def test_in_place_and_repeatable(lp):
    g = [gradient((70, 90), 1), gradient((2, 64, 30), 2), gradient((300, 300), 4)]
    outs = lp.orthogonalize(g)
    assert all(torch.equal(a, b) for a, b in zip(outs, lp.orthogonalize(g)))
    ws = torch.empty(lp.lp_orthogonalize_workspace_bytes(g), dtype=torch.uint8, device="cuda").fill_(255)
    lp.lp_orthogonalize(g, g, ws)
    assert all(torch.equal(a, b) for a, b in zip(outs, g))


def test_empty_lists(lp):
    assert lp.orthogonalize([]) == []
    lp.muon_step([], [], [], lr=0.1)
    outs = lp.orthogonalize([torch.empty(0, 4, 4, device="cuda"), gradient((8, 8), 1), torch.empty(3, 0, device="cuda")])
    assert outs[0].shape == (0, 4, 4) and outs[2].shape == (3, 0)
    assert torch.equal(outs[1], lp.orthogonalize([gradient((8, 8), 1)])[0])


def test_streams_and_graphs(lp):
    mats = [gradient((64, 64), 1), gradient((2, 150, 70), 2)]
    outs = lp.orthogonalize(mats)
    ws = torch.empty(lp.lp_orthogonalize_workspace_bytes(mats), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lp.lp_orthogonalize(mats, outs, ws)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lp.lp_orthogonalize(mats, outs, ws)
    for seed in range(3):
        for t in mats:
            t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(seed)))
        want = lp.orthogonalize(mats)
        for t in outs:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_refusals(lp):
    g = gradient((80, 80), 1)   # (smaller ones need no workspace)
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")

    def status(f):
        with pytest.raises(lp.LightplaneError) as e:
            f()
        return e.value.status

    assert status(lambda: lp.lp_orthogonalize([g], [g], ws[:256])) == lp.LP_ERR_WORKSPACE
    assert status(lambda: lp.lp_orthogonalize([g], [g], ws[1:])) == lp.LP_ERR_INVALID_ARG
    for kw in (dict(steps=0), dict(steps=17), dict(eps=-1.0), dict(eps=float("inf")), dict(coeffs=(float("nan"), 0.0, 0.0)),
               dict(coeffs=(30.0, 0.0, 0.0)), dict(coeffs=(1.0, 50.0, 3.0))):
        assert status(lambda: lp.lp_orthogonalize([g], [g], ws, **kw)) == lp.LP_ERR_INVALID_ARG
    w = g.clone()
    for kw in (dict(lr=float("nan")), dict(lr=0.1, momentum=float("inf")), dict(lr=0.1, scale=3), dict(lr=0.1, nesterov=2)):
        assert status(lambda: lp.lp_muon_step([w], [g], [g.clone()], ws, **kw)) == lp.LP_ERR_INVALID_ARG
    assert torch.equal(w, g)
    for bad in (lambda: lp.orthogonalize([g.double()]), lambda: lp.orthogonalize([g.t()[1:]]), lambda: lp.orthogonalize([g[0]]),
                lambda: lp.orthogonalize([g.cpu()]), lambda: lp.lp_orthogonalize([g], [g.half()], ws),
                lambda: lp.lp_orthogonalize([g], [], ws), lambda: lp.muon_step([w.half()], [g], [g], lr=0.1),
                lambda: lp.muon_step([w], [g[:8]], [g], lr=0.1), lambda: lp.orthogonalize([g], steps=3, coeffs=[(1.0, 1.0, 1.0)])):
        with pytest.raises((ValueError, lp.LightplaneError)):
            bad()
