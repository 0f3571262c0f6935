"""The norms around a residual block, forward and backward, against the formulas in 64 bits (gradients by torch's derivatives of them).

Tolerances.  Means and variances are sums of C values over at most 16 values a lane, a tree of lanes and 8 waves: some 30 u (u = 2^-24) of the
sum of absolute values; a normed value carries that, the rounding of the difference to the mean (relative to the largest |s|) and some products:
TOL = 1e-5 of the largest value in the tensor covers it for values whose mean is of the size of their spread, and for gradients, which are
sums of three such terms.  Each result is rounded once: half a step of its type.  Column sums are sums over the positions of terms that
are good to TOL: TOL of the sum of the terms' absolute values.  A term d_y xh of d_gamma is good to TOL of |d_y| times the LARGEST |xh|, not of itself:
the difference to the mean (and s itself) is rounded at the size of s and of the mean, u (|s| + |mean|) rstd, also where xh is near zero."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TOL = 1e-5
TYPES = [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.float32, torch.float16), (torch.bfloat16, torch.bfloat16),
         (torch.float16, torch.float16)]
HALF = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
# samples, positions, channels
SIZES = [(1, 1, 512), (1, 1, 1), (1, 7, 2), (2, 5, 3), (3, 111, 72), (2, 64, 8), (1, 300, 32), (4, 33, 100), (2, 50, 65), (1, 40, 511), (2, 9, 513),
         (1, 12, 1024), (2, 3, 2047), (1, 5, 4096), (1, 3, 4099), (1, 2, 8192), (700, 2, 24), (1, 20000, 16), (5, 1, 264)]
OPTIONS = [dict(kind="rms", post=False, gate=None, alpha=1.0), dict(kind="layer", post=True, gate="channel", alpha=0.7),
           dict(kind="rms", post=True, gate="sample", alpha=1.0), dict(kind="layer", post=False, gate="sample", alpha=-1.5),
           dict(kind="rms", post=True, gate="channel", alpha=0.0)]


def _norm(v, kind, eps):
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
    return v / torch.sqrt(v.square().mean(-1, keepdim=True) + eps)


def _strided(t, extra, offset):
    if not extra:
        return t.cuda()
    wide = torch.full(t.shape[:-1] + (t.shape[-1] + extra,), float("nan"), dtype=t.dtype, device="cuda")
    out = wide[..., offset:offset + t.shape[-1]]
    out.copy_(t)
    return out


def _case(n, p, c, h_dtype, f_dtype, opt, seed, strided=(0, 0)):
    gen = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    put = lambda t, d: _strided(t.to(d), *strided)  # noqa: E731
    t = {"h": put(rand(n, p, c) + 0.4 * rand(c), h_dtype), "f": put(0.7 * rand(n, p, c) + 0.2, f_dtype),
         "d_s": put(0.1 * rand(n, p, c), h_dtype), "d_y": put(0.1 * rand(n, p, c), f_dtype),
         "gamma": (1 + 0.3 * rand(c)).cuda(), "beta": (0.3 * rand(c)).cuda(), "post_gamma": (1 + 0.3 * rand(c)).cuda() if opt["post"] else None,
         "gate": None if opt["gate"] is None else (0.5 + 0.4 * rand(*((n, c) if opt["gate"] == "sample" else (c,)))).cuda()}
    return t


def _lp_norm(lp, t, opt, eps=1e-5):
    return lp.ResidualNorm(lp.LP_NORM_LAYER if opt["kind"] == "layer" else lp.LP_NORM_RMS, t["gamma"], t["beta"], opt["post"], t["post_gamma"],
                           t["gate"], opt["alpha"], eps)


def _reference(t, opt, with_f=True, up_s=True, up_y=True, eps=1e-5):
    """Results and gradients in 64 bits, and the sums of absolute terms of the parameters' gradients."""
    leaf = {k: None if v is None else v.detach().double().cpu().requires_grad_(True) for k, v in t.items() if k not in ("d_s", "d_y")}
    h, f = leaf["h"], leaf["f"]
    gate = leaf["gate"]
    if gate is not None and gate.dim() == 2:
        gate_b = gate.unsqueeze(1)
    else:
        gate_b = gate
    s = opt["alpha"] * h
    fh = None
    if with_f:
        fh = _norm(f, opt["kind"], eps) if opt["post"] else f
        u = fh * leaf["post_gamma"] if opt["post"] else fh
        s = s + (u if gate is None else gate_b * u)
    xh = _norm(s, opt["kind"], eps)
    y = xh * leaf["gamma"] + leaf["beta"]
    loss = 0.0
    if up_s:
        loss = loss + (s * t["d_s"].double().cpu()).sum()
    if up_y:
        loss = loss + (y * t["d_y"].double().cpu()).sum()
    names = [k for k, v in leaf.items() if v is not None and (with_f or k in ("h", "gamma", "beta"))]
    grads = dict(zip(names, torch.autograd.grad(loss, [leaf[k] for k in names], allow_unused=True)))
    return s.detach(), y.detach(), {k: torch.zeros_like(leaf[k]) if v is None else v for k, v in grads.items()}, xh.detach(), None if fh is None else fh.detach()


def _close(got, want, label, dtype=torch.float32, floor=1e-3, scale=None):
    got, want = got.double().cpu(), want.double()
    assert got.shape == want.shape and torch.isfinite(got).all(), label
    if not want.numel():
        return
    size = torch.full((), max(float(want.abs().max()), floor), dtype=torch.float64) if scale is None else scale + 1e-9
    bound = TOL * size + HALF[dtype] * (want.abs() + TOL * size) + TINY[dtype]
    over = float(((got - want).abs() - bound).max())
    assert over <= 0, f"{label}: {float((got - want).abs().max())} off, {over} over its bound"


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("n,p,c", SIZES)
def test_forward_and_backward(lp, n, p, c, types):
    h_dtype, f_dtype = types
    for i, opt in enumerate(OPTIONS):
        # C = 1 and C = 2: a layer norm of one channel is its beta, of two channels +-1 almost everywhere: gradients are differences of
        # equal terms there, and only the forward says something
        t = _case(n, p, c, h_dtype, f_dtype, opt, 17 * n + p + c + i, [(0, 0), (5, 3), (0, 0), (16, 8), (0, 0)][i])
        norm = _lp_norm(lp, t, opt)
        s, y = lp.residual_norm_fwd(norm, t["h"], t["f"])
        want_s, want_y, grads, xh, fh = _reference(t, opt)
        assert s.dtype == h_dtype and y.dtype == f_dtype and s.stride() == t["h"].stride()
        _close(s, want_s, "s", h_dtype)
        if c > 2 or opt["kind"] == "rms":
            _close(y, want_y, "y", f_dtype)
        if c <= 3:
            continue
        d_h, d_f, d_gamma, d_beta, d_post_gamma, d_gate = lp.residual_norm_bwd(norm, t["h"], t["f"], t["d_s"], t["d_y"])
        _close(d_h, grads["h"], "d_h", h_dtype)
        _close(d_f, grads["f"], "d_f", f_dtype)
        d_y = t["d_y"].double().cpu()
        _close(d_gamma, grads["gamma"], "d_gamma", scale=d_y.abs().sum((0, 1)) * xh.abs().max())
        _close(d_beta, grads["beta"], "d_beta", scale=d_y.abs().sum((0, 1)))
        # g of the formulas, with the error of its terms' size
        terms = fh.abs() * float(grads["f"].abs().max() + grads["h"].abs().max() + t["d_s"].double().abs().max() + 3 * t["d_y"].double().abs().max())
        if opt["post"]:
            _close(d_post_gamma, grads["post_gamma"], "d_post_gamma", scale=terms.sum((0, 1)))
        if opt["gate"]:
            _close(d_gate, grads["gate"], "d_gate", scale=2 * (terms.sum(1) if opt["gate"] == "sample" else terms.sum((0, 1))))
        assert (d_post_gamma is None) == (not opt["post"]) and (d_gate is None) == (opt["gate"] is None)


@pytest.mark.parametrize("c", [24, 65, 1000])
def test_parts_of_the_block(lp, c):
    """Without a block's result, without a norm, without one of the upstream gradients, and with gradients that are not wanted."""
    opt = OPTIONS[2]
    t = _case(3, 50, c, torch.float32, torch.float32, opt, c)
    norm = _lp_norm(lp, t, opt)
    # the first norm of a network
    s, y = lp.residual_norm_fwd(norm, t["h"])
    assert s is t["h"]
    _, want_y, grads, _, _ = _reference(t, opt, with_f=False)
    _close(y, want_y, "y")
    d_h, d_f, d_gamma, d_beta, d_post_gamma, d_gate = lp.residual_norm_bwd(norm, t["h"], None, t["d_s"], t["d_y"])
    _close(d_h, grads["h"], "d_h")
    assert d_f is None and d_post_gamma is None and d_gate is None
    scaled = lp.ResidualNorm(lp.LP_NORM_LAYER, t["gamma"], t["beta"], alpha=0.5)
    s, y = lp.residual_norm_fwd(scaled, t["h"])
    assert torch.equal(s, 0.5 * t["h"])
    # the sum alone
    s, y = torch.empty_like(t["h"]), torch.empty_like(t["f"])
    lp.lp_residual_norm_fwd(norm, t["h"], t["f"], s, None)
    want_s = _reference(t, opt)[0]
    _close(s, want_s, "s")
    lp.lp_residual_norm_fwd(norm, t["h"], t["f"], None, y)
    _close(y, _reference(t, opt)[1], "y")
    # upstream gradients that are not there
    for up_s, up_y in ((True, False), (False, True), (False, False)):
        grads = _reference(t, opt, up_s=up_s, up_y=up_y)[2] if up_s or up_y else {k: torch.zeros_like(t[k].cpu().double()) for k in ("h", "f")}
        got = lp.residual_norm_bwd(norm, t["h"], t["f"], t["d_s"] if up_s else None, t["d_y"] if up_y else None)
        _close(got[0], grads["h"], "d_h")
        _close(got[1], grads["f"], "d_f")
    whole = lp.residual_norm_bwd(norm, t["h"], t["f"], t["d_s"], t["d_y"])
    ws = torch.empty(lp.lp_residual_norm_workspace_bytes(norm, t["h"]), dtype=torch.uint8, device="cuda")
    for wanted in range(64):
        outs = [torch.zeros_like(g) if wanted >> i & 1 else None for i, g in enumerate(whole)]
        lp.lp_residual_norm_bwd(norm, t["h"], t["f"], t["d_s"], t["d_y"], *outs, ws)
        assert all(o is None or torch.equal(o, g) for o, g in zip(outs, whole)), wanted


@pytest.mark.parametrize("opt", OPTIONS, ids=lambda o: f"{o['kind']}-{o['post']}-{o['gate']}")
def test_gradients_against_differences(lp, opt):
    """The backward's gradients are the slopes of the formulas along random directions (differences in 64 bits, good to the square of their step)."""
    t = _case(3, 20, 40, torch.float32, torch.float32, opt, 12)
    norm = _lp_norm(lp, t, opt)
    got = dict(zip(("h", "f", "gamma", "beta", "post_gamma", "gate"), lp.residual_norm_bwd(norm, t["h"], t["f"], t["d_s"], t["d_y"])))
    host = {k: v.double().cpu() for k, v in t.items() if v is not None}

    def loss(values):
        u = {**host, **values}
        s, y = _reference({**u, **{k: None for k in t if k not in u}}, opt)[:2]
        return float((s * u["d_s"]).sum() + (y * u["d_y"]).sum())

    gen = torch.Generator().manual_seed(13)
    names = [k for k, g in got.items() if g is not None]
    for _ in range(4):
        way = {k: torch.randn(host[k].shape, generator=gen).double() for k in names}
        slope = (loss({k: host[k] + 1e-5 * way[k] for k in names}) - loss({k: host[k] - 1e-5 * way[k] for k in names})) / 2e-5
        terms = [got[k].double().cpu() * way[k] for k in names]
        # (fp32 gradients are good to TOL of the largest; the differences' own error is some 1e-8)
        bound = sum(TOL * float(got[k].abs().max()) * way[k].numel() ** 0.5 * 3 for k in names) + 1e-6
        assert abs(sum(float(v.sum()) for v in terms) - slope) <= bound


def test_in_place_and_accumulation(lp):
    opt = OPTIONS[1]
    t = _case(2, 90, 72, torch.bfloat16, torch.bfloat16, opt, 1)
    norm = _lp_norm(lp, t, opt)
    t = {k: None if v is None else v.contiguous() for k, v in t.items()}
    s, y = lp.residual_norm_fwd(norm, t["h"], t["f"])
    whole = lp.residual_norm_bwd(norm, t["h"], t["f"], t["d_s"], t["d_y"])
    h, f = t["h"].clone(), t["f"].clone()
    lp.lp_residual_norm_fwd(norm, h, f, h, f)
    assert torch.equal(h, s) and torch.equal(f, y)
    ws = torch.empty(lp.lp_residual_norm_workspace_bytes(norm, t["h"]), dtype=torch.uint8, device="cuda")
    before = [torch.randn_like(g) for g in whole[2:]]
    params = [b.clone() for b in before]
    d_s, d_y = t["d_s"].clone(), t["d_y"].clone()
    lp.lp_residual_norm_bwd(norm, t["h"], t["f"], d_s, d_y, d_s, d_y, *params, ws)
    assert torch.equal(d_s, whole[0]) and torch.equal(d_y, whole[1])
    for got, b, g in zip(params, before, whole[2:]):
        assert torch.allclose(got, b + g, rtol=2.0 ** -22, atol=0)


def test_rows_that_are_not_finite_and_rows_of_zeros(lp):
    for c in (24, 65, 700):
        opt = OPTIONS[1]
        t = _case(1, 40, c, torch.float32, torch.float32, opt, 2)
        t = {k: None if v is None else v.contiguous() for k, v in t.items()}
        norm = _lp_norm(lp, t, opt)
        s, y = lp.residual_norm_fwd(norm, t["h"], t["f"])
        d_h, d_f = lp.residual_norm_bwd(norm, t["h"], t["f"], t["d_s"], t["d_y"])[:2]
        h = t["h"].clone()
        h[0, 7, c - 1], h[0, 11, 0] = float("nan"), float("inf")
        keep = torch.ones(40, dtype=torch.bool, device="cuda")
        keep[[7, 11]] = False
        s2, y2 = lp.residual_norm_fwd(norm, h, t["f"])
        got = lp.residual_norm_bwd(norm, h, t["f"], t["d_s"], t["d_y"])
        for a, b in ((s, s2), (y, y2), (d_h, got[0]), (d_f, got[1])):
            assert torch.equal(a[0, keep], b[0, keep])
        assert torch.isnan(y2[0, 7]).all()
        # rows of zeros: norm(0) = 0
        zero = torch.zeros_like(t["h"])
        s, y = lp.residual_norm_fwd(norm, zero, zero)
        assert not s.any() and torch.equal(y, t["beta"].expand_as(y))
        assert all(torch.isfinite(g).all() for g in lp.residual_norm_bwd(norm, zero, zero, t["d_s"], t["d_y"]))


def test_a_large_mean_does_not_cancel_the_variance(lp):
    gen = torch.Generator().manual_seed(3)
    x = (1000 + torch.randn(1, 64, 256, generator=gen)).cuda()
    _, y = lp.residual_norm_fwd(lp.ResidualNorm(lp.LP_NORM_LAYER), x)
    want = _norm(x.double().cpu(), "layer", 1e-5)
    # values near 1000 differ from their mean by a rounding of the mean of 2^-24 1000 = 6e-5, and the spread is 1
    assert float((y.double().cpu() - want).abs().max()) < 5e-4


def test_many_samples_and_no_positions(lp):
    opt = OPTIONS[2]
    t = _case(9000, 1, 40, torch.float32, torch.bfloat16, opt, 4)
    norm = _lp_norm(lp, t, opt)
    got = lp.residual_norm_bwd(norm, t["h"], t["f"], t["d_s"], t["d_y"])
    _, _, grads, _, fh = _reference(t, opt)
    _close(got[5], grads["gate"], "d_gate")
    _close(got[4], grads["post_gamma"], "d_post_gamma", scale=(fh.abs() * 2).sum((0, 1)))
    empty = t["h"][:, :0]
    s, y = lp.residual_norm_fwd(norm, empty, t["f"][:, :0])
    assert s.shape == y.shape == (9000, 0, 40)
    got = lp.residual_norm_bwd(norm, empty, t["f"][:, :0], None, None)
    assert not any(g.any() for g in got)


def test_offsets_beyond_32_bits(lp):
    n, c = (1 << 25) + 3, 64
    h = torch.zeros(1, n, c, dtype=torch.bfloat16, device="cuda")
    rows = [0, 1 << 24, n - 1]
    gen = torch.Generator().manual_seed(5)
    h[0, rows] = torch.randn(3, c, generator=gen).to(torch.bfloat16).cuda()
    norm = lp.ResidualNorm(lp.LP_NORM_RMS)
    _, y = lp.residual_norm_fwd(norm, h, torch.zeros_like(h))
    want = lp.residual_norm_fwd(norm, h[:, rows].contiguous(), torch.zeros(1, 3, c, dtype=torch.bfloat16, device="cuda"))[1]
    assert torch.equal(y[0, rows], want[0])
    y[0, rows] = 0
    assert not y.any()


@pytest.mark.parametrize("c", [61, 600])
def test_more_than_the_cache_holds(lp, c):
    """Results of such calls are stored another way; rows of odd sizes.  A position's result does not depend on the others."""
    p = 300_000_000 // (8 * c) + 77
    gen = torch.Generator(device="cuda").manual_seed(2)
    h, f, d_s, d_y = (torch.randn(1, p, c, generator=gen, device="cuda").bfloat16() for _ in range(4))
    norm = lp.ResidualNorm(lp.LP_NORM_LAYER, torch.randn(c, generator=gen, device="cuda"), torch.randn(c, generator=gen, device="cuda"), True)
    s, y = lp.residual_norm_fwd(norm, h, f)
    d_h, d_f = lp.residual_norm_bwd(norm, h, f, d_s, d_y)[:2]
    for rows in torch.arange(p, device="cuda").split(p // 4 + 1):
        rows = slice(int(rows[0]), int(rows[-1]) + 1)
        part = lp.residual_norm_fwd(norm, h[:, rows], f[:, rows])
        grads = lp.residual_norm_bwd(norm, h[:, rows], f[:, rows], d_s[:, rows], d_y[:, rows])
        for a, b in ((s, part[0]), (y, part[1]), (d_h, grads[0]), (d_f, grads[1])):
            assert torch.equal(a[:, rows], b)


def test_captured_and_replayed(lp):
    opt = OPTIONS[2]
    t = _case(6, 200, 96, torch.float32, torch.bfloat16, opt, 6)
    norm = _lp_norm(lp, t, opt)

    def step():
        return (*lp.residual_norm_fwd(norm, t["h"], t["f"]), *lp.residual_norm_bwd(norm, t["h"], t["f"], t["d_s"], t["d_y"]))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(4):
        t["h"].copy_(torch.randn_like(t["h"]))
        t["d_y"].copy_(torch.randn_like(t["d_y"]))
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))
