"""Group norm with an activation, forward and backward, against the formulas in 64 bits.

Tolerances (u = 2^-24): a value of xh carries the rounding of x - mean, rstd and two products and the error of the sums behind
mean and rstd, a thread's sums of at most some thousand terms joined pairwise: some 1e-6 of the largest |xh| (at most 12 here);
the activation's exponential is good to some 1e-6 of its argument's size.  3e-5 of the outputs' largest value covers them; 16-bit outputs add half a unit in
their last place.  Gradients of the parameters are sums over N P terms whose rounding errors are relative to the terms: 3e-5 of the sum
of their absolute values."""
import math


import pytest
import torch

pytestmark = pytest.mark.gpu

TOL = 3e-5
HALF_ULP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
ACTS = ["none", "relu", "silu", "gelu"]


def _act(z, act):
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return z.clamp(min=0), (z > 0).double()
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return z * s, s + z * s * (1 - s)
    phi = 0.5 * (1 + torch.erf(z / math.sqrt(2)))
    return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)


def reference(x, groups, gamma, beta, act, eps, occ=None, d_y=None):
    """The formulas on the CPU in 64 bits, one (sample, group) after the other."""
    n, c = x.shape[0], x.shape[-1]
    xf = x.reshape(n, -1, c).double().cpu()
    p = xf.shape[1]
    on = torch.ones(n, p, dtype=torch.bool) if occ is None else occ.reshape(n, p).cpu() > 0
    gamma = torch.ones(c).double() if gamma is None else gamma.double().cpu()
    beta = torch.zeros(c).double() if beta is None else beta.double().cpu()
    y, dx = torch.zeros_like(xf), torch.zeros_like(xf)
    dg, db, dg_abs, db_abs = (torch.zeros(c).double() for _ in range(4))
    stats = torch.zeros(n, groups, 2).double()
    size = c // groups
    up = None if d_y is None else d_y.reshape(n, p, c).double().cpu()
    for i in range(n):
        for g in range(groups):
            ch = slice(g * size, (g + 1) * size)
            v = xf[i, :, ch][on[i]]
            if v.numel() == 0:
                continue
            mean = v.mean()
            rstd = 1 / torch.sqrt(((v - mean) ** 2).mean() + eps)
            stats[i, g, 0], stats[i, g, 1] = mean, rstd
            xh = (v - mean) * rstd
            out, slope = _act(xh * gamma[ch] + beta[ch], act)
            y[i, :, ch][on[i]] = out
            if up is not None:
                gr = up[i, :, ch][on[i]] * slope
                dg[ch] += (gr * xh).sum(0)
                db[ch] += gr.sum(0)
                dg_abs[ch] += (gr * xh).abs().sum(0)
                db_abs[ch] += gr.abs().sum(0)
                gg = gr * gamma[ch]
                dx[i, :, ch][on[i]] = rstd * (gg - gg.mean() - xh * (gg * xh).mean())
    shape = x.shape
    return y.view(shape), stats, dx.view(shape), dg, db, dg_abs, db_abs


def _close(got, want, tol, label, ulp=0.0):
    got = got.double().cpu()
    assert torch.isfinite(got).all(), label
    err = (got - want).abs()
    bound = tol * max(float(want.abs().max()), 1e-3) + ulp * want.abs() + (1e-7 if ulp > 1e-4 else 0.0)   # (16-bit types: their smallest steps)
    worst = float((err - bound).max()) if err.numel() else 0.0
    assert worst <= 0, f"{label}: {float(err.max())} off, {worst} over the bound"


def _inputs(shape, x_dtype, seed, mean=0.0, std=0.8):
    gen = torch.Generator().manual_seed(seed)
    x = (torch.randn(shape, generator=gen) * std + mean).to(x_dtype).cuda()
    c = shape[-1]
    return x, (1 + 0.3 * torch.randn(c, generator=gen)).cuda(), (0.3 * torch.randn(c, generator=gen)).cuda(), gen


def check(lp, x, groups, gamma, beta, act, gen, occ=None, y_dtype=None, eps=1e-5):
    y_dtype = y_dtype or x.dtype
    d_y = torch.randn(x.shape, generator=gen).to(y_dtype).cuda()
    if act == "relu":   # the gradient hangs on the sign of the argument: none is asked for where rounding could turn that
        z = reference(x, groups, gamma, beta, "none", eps, occ)[0]
        d_y[z.abs().cuda() < 1e-4] = 0
    y_ref, st_ref, dx_ref, dg_ref, db_ref, dg_abs, db_abs = reference(x, groups, gamma, beta, act, eps, occ, d_y)
    norm = lp.GroupNorm(groups, gamma, beta, getattr(lp, "LP_ACT_" + act.upper()), eps, occ)
    y, stats = lp.group_norm_fwd(norm, x, y_dtype)
    d_x, d_gamma, d_beta = lp.group_norm_bwd(norm, x, stats, d_y)
    torch.cuda.synchronize()
    assert y.dtype == y_dtype and d_x.dtype == x.dtype
    assert float(((stats[..., 0].double().cpu() - st_ref[..., 0]).abs() - 1e-7 * st_ref[..., 0].abs()).max()) <= 2e-6, "mean"
    _close(stats[..., 1], st_ref[..., 1], 1e-5, "rstd")
    _close(y, y_ref, TOL, "y", HALF_ULP[y_dtype])
    _close(d_x, dx_ref, TOL, "d_x", HALF_ULP[x.dtype])
    assert float(((d_gamma.double().cpu() - dg_ref).abs() - TOL * dg_abs - 1e-6).max()) <= 0
    assert float(((d_beta.double().cpu() - db_ref).abs() - TOL * db_abs - 1e-6).max()) <= 0
    return norm, y, stats, d_y, d_x, d_gamma, d_beta


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("types", [("f32", "f32"), ("f32", "bf16"), ("f32", "f16"), ("bf16", "bf16"), ("f16", "f16")])
@pytest.mark.parametrize("shape,groups", [((1, 1024, 16), 4), ((2, 37, 41, 48), 6), ((3, 301, 9), 3), ((2, 1, 32), 2), ((1, 5, 5, 7, 30), 5)])
def test_against_64_bits(lp, act, types, shape, groups):
    t = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
    x, gamma, beta, gen = _inputs(shape, t[types[0]], 11 + len(shape))
    check(lp, x, groups, gamma, beta, act, gen, y_dtype=t[types[1]])


@pytest.mark.parametrize("channels,groups", [(1, 1), (2, 2), (3, 1), (6, 2), (12, 3), (33, 11), (320, 32), (1028, 4), (2051, 1)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_channel_counts(lp, channels, groups, dtype):
    x, gamma, beta, gen = _inputs((2, 77, channels), dtype, channels)
    check(lp, x, groups, gamma, beta, "silu", gen)


@pytest.mark.parametrize("p", [2, 3, 255, 256, 4097, 70001])
def test_lengths(lp, p):
    x, gamma, beta, gen = _inputs((2, p, 8), torch.float32, p)
    check(lp, x, 2, gamma, beta, "silu", gen)


def test_many_samples(lp):
    x, gamma, beta, gen = _inputs((3000, 5, 16), torch.float32, 5)
    check(lp, x, 4, gamma, beta, "gelu", gen)


def test_without_parameters(lp):
    x, _, _, gen = _inputs((2, 100, 16), torch.bfloat16, 3)
    check(lp, x, 4, None, None, "silu", gen)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shape,groups", [((3, 9, 8, 11, 16), 4), ((2, 1000, 6), 2), ((4, 4099, 32), 8)])
def test_occupancy(lp, dtype, shape, groups):
    """Cells that nothing landed in are no part of it, whatever they hold; a sample without any cell is zeros."""
    x, gamma, beta, gen = _inputs(shape, dtype, 21)
    occ = (torch.rand(shape[:-1], generator=gen) - 0.8).clamp(min=0).cuda()
    occ[1] = 0
    occ.view(-1)[3] = float("nan")   # (not above zero)
    occ.view(-1)[4] = -1.0
    occ.view(-1)[5] = float("inf")
    off = ~(occ > 0)
    x[off] = 0
    d_y_poison = off
    x_poisoned = x.clone()
    x_poisoned[off] = float("nan")
    norm, y, stats, d_y, d_x, d_gamma, d_beta = check(lp, x, groups, gamma, beta, "silu", gen, occ=occ)
    assert (y[off] == 0).all() and (d_x[off] == 0).all() and (stats[1] == 0).all()
    d_y = d_y.clone()
    d_y[d_y_poison] = float("inf")
    y2, stats2 = lp.group_norm_fwd(norm, x_poisoned)
    d_x2, d_gamma2, d_beta2 = lp.group_norm_bwd(norm, x_poisoned, stats2, d_y)
    for a, b in ((y, y2), (stats, stats2), (d_x, d_x2), (d_gamma, d_gamma2), (d_beta, d_beta2)):
        assert torch.equal(a, b)


def test_mean_far_from_zero(lp):
    """A mean of 100 standard deviations does not cost the variance its digits (fp32 values near 80 are 8e-6 apart: 1e-5 of
    the deviation, which x itself carries)."""
    x, gamma, beta, gen = _inputs((2, 5000, 16), torch.float32, 8, mean=80.0)
    check(lp, x, 4, gamma, beta, "none", gen)


def test_constant_input(lp):
    """No variance: y = act(beta), rstd = eps^(-1/2), gradients are finite."""
    x = torch.full((1, 500, 8), 3.25, device="cuda")
    gamma, beta = torch.ones(8, device="cuda"), torch.full((8,), 0.5, device="cuda")
    norm = lp.GroupNorm(2, gamma, beta, lp.LP_ACT_NONE, 1e-4)
    y, stats = lp.group_norm_fwd(norm, x)
    assert torch.equal(y, torch.full_like(y, 0.5)) and torch.allclose(stats[..., 1], torch.full((1, 2), 100.0, device="cuda"))
    d_x, d_gamma, d_beta = lp.group_norm_bwd(norm, x, stats, torch.ones_like(x))
    assert float(d_x.abs().max()) <= 1e-4 and float(d_gamma.abs().max()) == 0 and torch.equal(d_beta, torch.full((8,), 500.0, device="cuda"))


def test_infinities_stay_in_their_group(lp):
    x, gamma, beta, _ = _inputs((2, 300, 16), torch.float32, 4)
    want, _ = lp.group_norm_fwd(lp.GroupNorm(4, gamma, beta, lp.LP_ACT_SILU), x)
    x[1, 17, 5] = float("inf")
    y, _ = lp.group_norm_fwd(lp.GroupNorm(4, gamma, beta, lp.LP_ACT_SILU), x)
    assert torch.isnan(y[1, :, 4:8]).all()
    y[1, :, 4:8] = want[1, :, 4:8]
    assert torch.equal(y, want)


def test_gradients_against_differences(lp):
    """The forward's own differences: sum(y w) for x, gamma, beta moved along random directions."""
    x, gamma, beta, gen = _inputs((2, 40, 12), torch.float32, 6)
    w = torch.randn(x.shape, generator=gen).cuda()
    norm = lp.GroupNorm(3, gamma, beta, lp.LP_ACT_SILU)
    _, stats = lp.group_norm_fwd(norm, x)
    d_x, d_gamma, d_beta = lp.group_norm_bwd(norm, x, stats, w)
    h = 1e-2

    def value(dx, dg, db):
        y, _ = lp.group_norm_fwd(lp.GroupNorm(3, gamma + dg, beta + db, lp.LP_ACT_SILU), x + dx)
        return float((y.double() * w.double()).sum())

    for k in range(3):
        v = torch.randn([x.shape, gamma.shape, beta.shape][k], generator=gen).cuda()
        v = v / v.norm()
        args = [[torch.zeros((), device="cuda")] * 3 for _ in range(2)]
        args[0][k], args[1][k] = h * v, -h * v
        diff = (value(*args[0]) - value(*args[1])) / (2 * h)
        got = float((v.double() * (d_x, d_gamma, d_beta)[k].double()).sum())
        assert abs(diff - got) <= 2e-3 * max(1.0, float((d_x, d_gamma, d_beta)[k].norm())), (k, diff, got)   # (h^2 of the third derivative, fp32 sums / h)


def test_parameter_gradients_accumulate_and_repeat(lp):
    x, gamma, beta, gen = _inputs((3, 2000, 16), torch.float32, 9)
    d_y = torch.randn(x.shape, generator=gen).cuda()
    norm = lp.GroupNorm(4, gamma, beta, lp.LP_ACT_SILU)
    _, stats = lp.group_norm_fwd(norm, x)
    first = lp.group_norm_bwd(norm, x, stats, d_y)
    again = lp.group_norm_bwd(norm, x, stats, d_y)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    ws = torch.empty(lp.lp_group_norm_workspace_bytes(norm, x)[1], dtype=torch.uint8, device="cuda")
    d_gamma, d_beta = torch.full((16,), 2.0, device="cuda"), torch.full((16,), -3.0, device="cuda")
    lp.lp_group_norm_bwd(norm, x, stats, d_y, None, d_gamma, d_beta, ws)
    assert torch.allclose(d_gamma, first[1] + 2, rtol=1e-6, atol=1e-5) and torch.allclose(d_beta, first[2] - 3, rtol=1e-6, atol=1e-5)
    d_x = torch.empty_like(x)
    lp.lp_group_norm_bwd(norm, x, stats, d_y, d_x, None, None, ws)
    assert torch.equal(d_x, first[0])


def test_slices_of_wider_tensors_and_in_place(lp):
    """A slice of the channels (half of what two layers left side by side); x and d_y overwritten by y and d_x."""
    gen = torch.Generator().manual_seed(2)
    wide = torch.randn(2, 10, 11, 48, generator=gen).cuda()
    for at, c in ((16, 32), (3, 12), (0, 16), (4, 8)):
        x = wide[..., at:at + c]
        norm = lp.GroupNorm(4, None, None, lp.LP_ACT_SILU)
        y, stats = lp.group_norm_fwd(norm, x)
        y_dense, stats_dense = lp.group_norm_fwd(norm, x.contiguous())
        assert torch.allclose(y, y_dense, rtol=1e-5, atol=1e-6) and torch.allclose(stats, stats_dense, rtol=1e-5, atol=1e-6)
        d_y = torch.randn(2, 10, 11, 64, generator=gen).cuda()[..., 5:5 + c]
        d_x, d_gamma, _ = lp.group_norm_bwd(norm, x, stats, d_y)
        e_x, e_gamma, _ = lp.group_norm_bwd(norm, x.contiguous(), stats_dense, d_y.contiguous())
        assert torch.allclose(d_x, e_x, rtol=1e-5, atol=1e-5) and torch.allclose(d_gamma, e_gamma, rtol=1e-5, atol=1e-5)
        # a slice written: the rest of the tensor stays
        out = torch.full_like(wide, 7.0)
        ws = torch.empty(max(lp.lp_group_norm_workspace_bytes(norm, x)), dtype=torch.uint8, device="cuda")
        lp.lp_group_norm_fwd(norm, x, out[..., at:at + c], None, ws)
        assert torch.equal(out[..., at:at + c], y) and (out[..., :at] == 7).all() and (out[..., at + c:] == 7).all()
        xi, di = x.contiguous(), d_y.contiguous()
        lp.lp_group_norm_bwd(norm, xi, stats_dense, di, di, None, None, ws)
        assert torch.allclose(di, e_x, rtol=1e-5, atol=1e-5)
        lp.lp_group_norm_fwd(norm, xi, xi, None, ws)
        assert torch.equal(xi, y_dense)


def test_unaligned_tensors(lp):
    gen = torch.Generator().manual_seed(12)
    for dtype, off in ((torch.float32, 1), (torch.bfloat16, 1), (torch.float16, 2)):
        base = torch.randn(2 * 50 * 16 + 8, generator=gen).to(dtype).cuda()
        x = base[off:off + 1600].view(2, 50, 16)
        y, _ = lp.group_norm_fwd(lp.GroupNorm(4, None, None, lp.LP_ACT_SILU), x)
        want = reference(x, 4, None, None, "silu", 1e-5)[0]
        _close(y, want, TOL, "y", HALF_ULP[dtype])


def test_empty(lp):
    norm = lp.GroupNorm(2)
    for shape in ((0, 5, 4), (3, 0, 4)):
        x = torch.empty(shape, device="cuda")
        y, stats = lp.group_norm_fwd(norm, x)
        d_x, d_gamma, _ = lp.group_norm_bwd(norm, x, stats, y)
        assert y.shape == x.shape and d_x.shape == x.shape and float(d_gamma.abs().max()) == 0


def test_offsets_beyond_32_bits(lp):
    """The last positions of a tensor of more than 2^32 bytes, by the first and last rows' own formula."""
    p, c = (1 << 28) + 77, 8
    x = torch.zeros(1, p, c, device="cuda", dtype=torch.float16)
    gen = torch.Generator().manual_seed(1)
    tail = torch.randn(64, c, generator=gen).half().cuda()
    x[0, -64:] = tail
    norm = lp.GroupNorm(2, None, None, lp.LP_ACT_NONE)
    y, stats = lp.group_norm_fwd(norm, x)
    t = tail.double().view(64, 2, 4)
    n = p * 4
    mean = t.sum((0, 2)) / n
    rstd = 1 / torch.sqrt((t ** 2).sum((0, 2)) / n - mean ** 2 + 1e-5)
    want = ((t - mean.view(1, 2, 1)) * rstd.view(1, 2, 1)).view(64, c).half()
    assert torch.allclose(stats[0, :, 1].double(), rstd, rtol=1e-4)
    assert torch.allclose(y[0, -64:].double(), want.double(), rtol=2e-3, atol=1e-3) and torch.equal(y[0, 0], y[0, 5])


def test_other_streams_and_graphs(lp):
    x, gamma, beta, gen = _inputs((2, 3001, 16), torch.float32, 13)
    d_y = torch.randn(x.shape, generator=gen).cuda()
    norm = lp.GroupNorm(4, gamma, beta, lp.LP_ACT_SILU)
    y, stats = lp.group_norm_fwd(norm, x)
    d_x, d_gamma, d_beta = lp.group_norm_bwd(norm, x, stats, d_y)
    ws = torch.empty(max(lp.lp_group_norm_workspace_bytes(norm, x)), dtype=torch.uint8, device="cuda")

    def step(stream=None):
        lp.lp_group_norm_fwd(norm, x, y, stats, ws, stream)
        d_gamma.zero_()
        d_beta.zero_()
        lp.lp_group_norm_bwd(norm, x, stats, d_y, d_x, d_gamma, d_beta, ws, stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    outs = [y, stats, d_x, d_gamma, d_beta]
    for seed in range(3):
        x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(seed)))
        step()
        want = [t.clone() for t in outs]
        for t in outs:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_refusals(lp):
    x = torch.zeros(1, 10, 8, device="cuda")
    y, ws = torch.empty_like(x), torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    stats = torch.empty(1, 2, 2, device="cuda")

    def status(f):
        with pytest.raises(lp.LightplaneError) as e:
            f()
        return e.value.status

    fwd = lambda norm, x=x, y=y, w=ws: lambda: lp.lp_group_norm_fwd(norm, x, y, None, w)  # noqa: E731
    assert status(fwd(lp.GroupNorm(3))) == lp.LP_ERR_INVALID_ARG
    assert status(fwd(lp.GroupNorm(0))) == lp.LP_ERR_INVALID_ARG
    assert status(fwd(lp.GroupNorm(2, act=4))) == lp.LP_ERR_INVALID_ARG
    assert status(fwd(lp.GroupNorm(2, eps=-1.0))) == lp.LP_ERR_INVALID_ARG
    assert status(fwd(lp.GroupNorm(2, eps=float("nan")))) == lp.LP_ERR_INVALID_ARG
    big = torch.zeros(1, 9000, 8, device="cuda")   # (smaller ones need no workspace)
    assert status(fwd(lp.GroupNorm(2), x=big, y=big.clone(), w=ws[:64])) == lp.LP_ERR_WORKSPACE
    assert status(fwd(lp.GroupNorm(2), x=big, y=big.clone(), w=None)) == lp.LP_ERR_WORKSPACE
    assert status(fwd(lp.GroupNorm(2), x=big, y=big.clone(), w=ws[1:])) == lp.LP_ERR_INVALID_ARG
    assert status(fwd(lp.GroupNorm(2), x=x.half(), y=y)) == lp.LP_ERR_UNSUPPORTED
    for bad in (lambda: lp.lp_group_norm_fwd(lp.GroupNorm(2), x.double(), y, None, ws),
                lambda: lp.lp_group_norm_fwd(lp.GroupNorm(2), x.cpu(), y, None, ws),
                lambda: lp.lp_group_norm_fwd(lp.GroupNorm(2), x.transpose(1, 2), y.transpose(1, 2), None, ws),
                lambda: lp.lp_group_norm_fwd(lp.GroupNorm(2), x, y[:, :5], None, ws),
                lambda: lp.lp_group_norm_fwd(lp.GroupNorm(2, torch.ones(7, device="cuda")), x, y, None, ws),
                lambda: lp.lp_group_norm_fwd(lp.GroupNorm(2, occupancy=torch.ones(1, 9, device="cuda")), x, y, None, ws),
                lambda: lp.lp_group_norm_fwd(lp.GroupNorm(2), x, y, stats[..., :1], ws),
                lambda: lp.lp_group_norm_bwd(lp.GroupNorm(2), x, stats, y, y.half(), None, None, ws),
                lambda: lp.lp_group_norm_fwd(lp.GroupNorm(2), x, x.view(-1)[:79].as_strided((1, 10, 8), (80, 8, 1), 0).view(torch.bfloat16)[..., :8], None, ws)):
        with pytest.raises((ValueError, lp.LightplaneError)):
            bad()
