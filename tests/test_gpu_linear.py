"""Products with bias, activation and residual, forward and backward, against the formulas in 64 bits.

Tolerances.  u = 2^-24.  A sum over K products adds 16 (16-bit types) or 2 (fp32) of them at a time to an fp32 accumulator, so K / 16 or
K / 2 additions follow one another and a result is off by at most that many times 2 u of the sum of the products' absolute values (2 u, not u:
the matrix cores need not round to nearest), plus some 16 for the additions inside a step.  The activations and their slopes are good to 5e-6 of
their argument's size, their slopes are at most 1.13.  A result is rounded once, by half a step of its type.  In d_x a 16-bit d_z is rounded by half a step
as well; in d_W what its parts leave is at most half a step of half a step in bf16; in fp16 the second part is bf16 and meets x rounded to bf16: half a step of
fp16 times two half steps of bf16."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

HALF = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}   # half a step
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}
ACT_TOL = 5e-6
ACTS = ["none", "relu", "silu", "gelu"]
DTYPES = [torch.float32, torch.bfloat16, torch.float16]
SIZES = [(1, 512, 2048), (1, 3, 5), (2, 4099, 7), (3, 72, 97), (8, 65, 33), (9, 64, 64), (16, 32, 32), (127, 31, 33), (128, 128, 128), (129, 129, 129),
         (1000, 72, 97), (4099, 16, 8), (300, 200, 1), (300, 1, 70), (257, 640, 384), (64, 2048, 512), (5000, 40, 130), (20011, 32, 128), (777, 64, 256),
         (600, 200, 136), (1030, 264, 520), (513, 530, 145), (515, 129, 131), (2000, 512, 64), (700, 1040, 40), (129, 128, 33), (1000, 64, 32), (333, 65, 128),
         (13, 1024, 256), (70, 515, 40), (300, 2048, 100), (150, 777, 300), (200, 100, 1100)]


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


def _sum_tol(k, dtype):
    return (k / (2 if dtype == torch.float32 else 16) + 16) * 2 * 2.0 ** -24


def _within(got, want, bound, label):
    got = got.double().cpu()
    assert torch.isfinite(got).all(), label
    over = ((got - want).abs() - bound).max() if got.numel() else torch.zeros(())
    assert float(over) <= 0, f"{label}: {float((got - want).abs().max())} off, {float(over)} over its bound"


def _strided(t, extra, offset):
    """The values of t as a slice of the channels of a wider tensor that holds NaN elsewhere."""
    if not extra:
        return t.cuda()
    wide = torch.full(t.shape[:-1] + (t.shape[-1] + extra,), float("nan"), dtype=t.dtype, device="cuda")
    out = wide[..., offset:offset + t.shape[-1]]
    out.copy_(t)
    return out


def _case(p, k, n, dtype, seed, strided=False):
    gen = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    extra, offset = ((5, 3) if strided == "odd" else (16, 8)) if strided else (0, 0)
    return {"x": _strided(rand(p, k).to(dtype), extra, offset), "w": (rand(n, k) / math.sqrt(k)).to(dtype).cuda(), "b": (0.3 * rand(n)).cuda(),
            "r": _strided(rand(p, n).to(dtype), extra, offset), "d_y": _strided((0.1 * rand(p, n)).to(dtype), extra, offset)}


def _act_id(lp, act):
    return {"none": lp.LP_ACT_NONE, "relu": lp.LP_ACT_RELU, "silu": lp.LP_ACT_SILU, "gelu": lp.LP_ACT_GELU}[act]


def _check_forward(t, act, dtype, y, pre, bias=True, residual=True):
    x, w = t["x"].double().cpu(), t["w"].double().cpu()
    k = x.shape[-1]
    z, size = x @ w.T, x.abs() @ w.abs().T
    if bias:
        z, size = z + t["b"].double().cpu(), size + t["b"].double().cpu().abs()
    z_tol = _sum_tol(k, dtype) * size
    want, _ = _act(z, act)
    tol = 1.13 * z_tol + (0 if act in ("none", "relu") else ACT_TOL * (1 + z.abs()))
    if residual:
        want = want + t["r"].double().cpu()
        tol = tol + 2.0 ** -23 * want.abs()
    _within(y, want, tol + HALF[dtype] * (want.abs() + tol) + TINY[dtype], "y")
    if pre is not None:
        _within(pre, z, z_tol + HALF[dtype] * (z.abs() + z_tol) + TINY[dtype], "pre")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("p,k,n", SIZES)
def test_forward(lp, p, k, n, dtype):
    for i, act in enumerate(ACTS):
        t = _case(p, k, n, dtype, 7 * p + k + n + i, ["", "odd", "even", ""][(i + p) % 4])
        full = (i + n) % 2 == 0
        lin = lp.Linear(t["w"], t["b"] if full or i < 2 else None, _act_id(lp, act))
        y, pre = lp.linear_fwd(lin, t["x"], t["r"] if full else None, keep=i % 2 == 0)
        assert y.dtype == dtype and y.shape == (p, n)
        _check_forward(t, act, dtype, y, pre, lin.bias is not None, full)


def _check_backward(t, act, dtype, pre, d_x, d_w, d_b, w0=None, b0=None):
    x, w, dy = t["x"].double().cpu(), t["w"].double().cpu(), t["d_y"].double().cpu()
    p, k = x.shape
    n = w.shape[0]
    dz, dz_tol = dy, torch.zeros_like(dy)
    if act != "none":
        z = pre.double().cpu()
        dz = dy * _act(z, act)[1]
        dz_tol = dy.abs() * (0 if act == "relu" else ACT_TOL) * (1 + z.abs()) + 2.0 ** -23 * dz.abs()
    rounded = 0.0 if act == "none" else HALF[dtype]
    want = dz @ w
    tol = (dz_tol + rounded * (dz.abs() + dz_tol) + TINY[dtype]) @ w.abs() + _sum_tol(n, dtype) * (dz.abs() @ w.abs())
    _within(d_x, want, 1.01 * (tol + HALF[dtype] * (want.abs() + tol)) + TINY[dtype], "d_x")
    # (up to 768 parts of the positions are added up, 12 one after the other in 64 lanes)
    left = 0.0 if act == "none" or dtype == torch.float32 else HALF[dtype] * HALF[torch.bfloat16] * (2.01 if dtype == torch.float16 else 1)
    want = dz.T @ x
    tol = (dz_tol + left * dz.abs()).T @ x.abs() + (2 * _sum_tol(p, dtype) + 64 * 2.0 ** -24) * (dz.abs().T @ x.abs())
    if w0 is not None:
        want, tol = want + w0.double().cpu(), tol + 2.0 ** -23 * (want.abs() + w0.double().cpu().abs())
    _within(d_w, want, 1.01 * tol + 1e-30, "d_weight")
    if d_b is not None:
        want, tol = dz.sum(0), dz_tol.sum(0) + (p / 8 + 64) * 2.0 ** -24 * dz.abs().sum(0)
        if b0 is not None:
            want, tol = want + b0.double().cpu(), tol + 2.0 ** -23 * (want.abs() + b0.double().cpu().abs())
        _within(d_b, want, 1.01 * tol + 1e-30, "d_bias")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("p,k,n", SIZES)
def test_backward(lp, p, k, n, dtype):
    for i, act in enumerate(ACTS):
        t = _case(p, k, n, dtype, 3 * p + k + n + i, ["odd", "", "even", ""][(i + p) % 4])
        pre = None
        if act != "none":
            pre = (t["x"].double().cpu() @ t["w"].double().cpu().T + t["b"].double().cpu()).to(dtype).cuda()
        lin = lp.Linear(t["w"], t["b"] if i % 2 == 0 else None, _act_id(lp, act))
        d_x, d_w, d_b = lp.linear_bwd(lin, t["x"], pre, t["d_y"])
        assert d_x.dtype == dtype and d_x.stride() == t["x"].stride() and d_w.dtype == torch.float32
        assert (d_b is None) == (lin.bias is None)
        _check_backward(t, act, dtype, pre, d_x, d_w, d_b)


@pytest.mark.parametrize("dtype", DTYPES)
def test_gradients_against_differences(lp, dtype):
    """The backward's gradients are the slopes of the forward: fp32 differences of a smooth loss along random directions."""
    t = _case(40, 24, 36, torch.float32, 5)
    if dtype != torch.float32:
        t = {k: v if k == "b" else v.to(dtype) for k, v in t.items()}
    lin = lp.Linear(t["w"], t["b"], lp.LP_ACT_SILU)
    _, pre = lp.linear_fwd(lin, t["x"], keep=True)
    d_x, d_w, d_b = lp.linear_bwd(lin, t["x"], pre, t["d_y"])
    gen = torch.Generator().manual_seed(1)

    def loss(x, w, b):   # the forward's formula, in 64 bits
        z = x @ w.T + b
        return float((_act(z, "silu")[0] * t["d_y"].double().cpu()).sum())

    x, w, b = (t[k].double().cpu() for k in ("x", "w", "b"))
    for _ in range(4):
        vx, vw, vb = (torch.randn(s.shape, generator=gen).double() for s in (x, w, b))
        step = 1e-5
        slope = (loss(x + step * vx, w + step * vw, b + step * vb) - loss(x - step * vx, w - step * vw, b - step * vb)) / (2 * step)
        got = sum(float((g.double().cpu() * v).sum()) for g, v in ((d_x, vx), (d_w, vw), (d_b, vb)))
        size = sum(float((g.double().cpu() * v).norm()) for g, v in ((d_x, vx), (d_w, vw), (d_b, vb)))
        # pre, d_z and d_x are rounded independently of the directions (3 sigma of three roundings); differences are good to step^2
        assert abs(got - slope) <= (3 * 3 * HALF[dtype] + 1e-6) * size


def test_what_is_written_and_what_is_not(lp):
    """Outputs that are slices of wider tensors: nothing beside them changes.  Gradients of the parameters are added to what is there."""
    p, k, n = 133, 31, 45
    for dtype in DTYPES:
        t = _case(p, k, n, dtype, 11, "odd")
        lin = lp.Linear(t["w"], t["b"], lp.LP_ACT_GELU)
        wide = torch.full((p + 2, n + 9), 7.0, dtype=dtype, device="cuda")
        y, pre = wide[1:-1, 4:4 + n], torch.empty(p, n, dtype=dtype, device="cuda")
        lp.lp_linear_fwd(lin, t["x"], y, pre, t["r"])
        _check_forward(t, "gelu", dtype, y, pre)
        wide[1:-1, 4:4 + n] = 7.0
        assert bool((wide == 7.0).all())
        d_wide = torch.full((p, k + 5), 3.0, dtype=dtype, device="cuda")
        d_x = d_wide[:, 3:3 + k]
        w0, b0 = torch.randn(n, k, device="cuda"), torch.randn(n, device="cuda")
        d_w, d_b = w0.clone(), b0.clone()
        ws = torch.empty(lp.lp_linear_workspace_bytes(lin, t["x"])[1], dtype=torch.uint8, device="cuda")
        lp.lp_linear_bwd(lin, t["x"], pre, t["d_y"], d_x, d_w, d_b, ws)
        _check_backward(t, "gelu", dtype, pre, d_x, d_w, d_b, w0, b0)
        d_wide[:, 3:3 + k] = 3.0
        assert bool((d_wide == 3.0).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_some_of_the_gradients(lp, dtype):
    t = _case(700, 33, 140, dtype, 2)
    lin = lp.Linear(t["w"], t["b"], lp.LP_ACT_SILU)
    _, pre = lp.linear_fwd(lin, t["x"], keep=True)
    whole = lp.linear_bwd(lin, t["x"], pre, t["d_y"])
    ws = torch.empty(lp.lp_linear_workspace_bytes(lin, t["x"])[1], dtype=torch.uint8, device="cuda")
    for wanted in range(8):
        outs = [torch.empty_like(t["x"]), torch.zeros_like(whole[1]), torch.zeros_like(whole[2])]
        outs = [o if wanted >> i & 1 else None for i, o in enumerate(outs)]
        lp.lp_linear_bwd(lin, t["x"], pre, t["d_y"], *outs, ws)
        for got, want in zip(outs, whole):
            assert got is None or torch.equal(got, want)


def test_residual_in_place_and_no_positions(lp):
    t = _case(300, 48, 64, torch.bfloat16, 3)
    lin = lp.Linear(t["w"], t["b"], lp.LP_ACT_RELU)
    want, _ = lp.linear_fwd(lin, t["x"], t["r"])
    y = t["r"].clone()
    version = y._version
    lp.lp_linear_fwd(lin, t["x"], y, None, y)
    assert torch.equal(y, want) and y._version > version
    y, pre = lp.linear_fwd(lin, t["x"][:0], keep=True)
    assert y.shape == pre.shape == (0, 64)
    d_x, d_w, d_b = lp.linear_bwd(lin, t["x"][:0], pre, y)
    assert d_x.shape == (0, 48) and not d_w.any() and not d_b.any()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("p,k,n", [(6, 65, 40), (200, 65, 40), (200, 32, 32)])
def test_values_that_are_not_finite_stay_in_their_rows(lp, p, k, n, dtype):
    """Rows of 65 channels: a chunk behind a row's end holds the next row's values, which must not meet a zero weight."""
    t = _case(p, k, n, dtype, 8)
    bad = torch.zeros(p, dtype=torch.bool)
    bad[[1, p // 2, p - 1]] = True
    x = t["x"].clone()
    x[bad.cuda(), 0] = torch.tensor([float("nan"), float("inf"), float("-inf")], device="cuda").to(dtype)
    lin = lp.Linear(t["w"], t["b"], lp.LP_ACT_NONE)
    y, want = lp.linear_fwd(lin, x)[0], lp.linear_fwd(lin, t["x"])[0]
    assert torch.equal(y[~bad.cuda()], want[~bad.cuda()])
    assert not torch.isfinite(y[bad.cuda()]).any()
    dy = t["d_y"].clone()
    dy[bad.cuda(), 0] = float("nan")
    d_x, d_w, _ = lp.linear_bwd(lin, t["x"], None, dy)
    clean = lp.linear_bwd(lin, t["x"], None, t["d_y"])
    assert torch.equal(d_x[~bad.cuda()], clean[0][~bad.cuda()]) and torch.isnan(d_x[bad.cuda()]).all()
    assert torch.isnan(d_w[0]).all() and torch.equal(d_w[1:], clean[1][1:])


def test_gradients_do_not_change_from_call_to_call(lp):
    t = _case(30000, 32, 96, torch.bfloat16, 4)
    lin = lp.Linear(t["w"], t["b"], lp.LP_ACT_GELU)
    _, pre = lp.linear_fwd(lin, t["x"], keep=True)
    first = lp.linear_bwd(lin, t["x"], pre, t["d_y"])
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, lp.linear_bwd(lin, t["x"], pre, t["d_y"])))


def test_offsets_beyond_32_bits(lp):
    """More than 2^32 bytes of x and of d_x; everything but a few rows is zero."""
    p, k, n = (1 << 25) + 77, 64, 8
    rows = torch.tensor([0, 1, (1 << 24) + 5, p - 2, p - 1])
    t = _case(len(rows), k, n, torch.bfloat16, 6)
    x, d_y = torch.zeros(p, k, dtype=torch.bfloat16, device="cuda"), torch.zeros(p, n, dtype=torch.bfloat16, device="cuda")
    x[rows.cuda()], d_y[rows.cuda()] = t["x"], t["d_y"]
    lin = lp.Linear(t["w"], None, lp.LP_ACT_NONE)
    y, _ = lp.linear_fwd(lin, x)
    t["r"] = None
    _check_forward(t, "none", torch.bfloat16, y[rows.cuda()], None, False, False)
    y[rows.cuda()] = 0
    assert not y.any()
    d_x, d_w, _ = lp.linear_bwd(lin, x, None, d_y)
    _check_backward(t, "none", torch.bfloat16, None, d_x[rows.cuda()], d_w, None)
    d_x[rows.cuda()] = 0
    assert not d_x.any()


@pytest.mark.parametrize("k,n,offset", [(16, 61, 0), (24, 264, 0), (16, 61, 3)])
def test_more_than_the_cache_holds(lp, k, n, offset):
    """Results of such calls are stored another way; rows of odd sizes, at odd addresses.  A position's result does not depend on the others."""
    p = 300_000_000 // (2 * (k + n)) + 77
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(p, k, generator=gen, device="cuda").bfloat16()
    lin = lp.Linear(torch.randn(n, k, generator=gen, device="cuda").bfloat16(), torch.randn(n, generator=gen, device="cuda"), lp.LP_ACT_SILU)
    wide = torch.full((p, n + 2 * offset), 5.0, dtype=torch.bfloat16, device="cuda")
    y = wide[:, offset:offset + n]
    ws = torch.empty(max(1, lp.lp_linear_workspace_bytes(lin, x)[0]), dtype=torch.uint8, device="cuda")
    lp.lp_linear_fwd(lin, x, y, None, None, ws)
    at = 0
    for rows in x.split(p // 4 + 1):
        assert torch.equal(y[at:at + len(rows)], lp.linear_fwd(lin, rows)[0])
        at += len(rows)
    if offset:
        assert bool((wide[:, :offset] == 5).all()) and bool((wide[:, offset + n:] == 5).all())


@pytest.mark.parametrize("p,k,n", [(3000, 72, 160), (700, 512, 136), (2000, 32, 64)])
def test_captured_and_replayed(lp, p, k, n):
    t = _case(p, k, n, torch.bfloat16, 9)
    lin = lp.Linear(t["w"], t["b"], lp.LP_ACT_GELU)

    def step():
        y, pre = lp.linear_fwd(lin, t["x"], t["r"], keep=True)
        return (y, *lp.linear_bwd(lin, t["x"], pre, t["d_y"]))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(4):
        t["x"].copy_(torch.randn_like(t["x"]))
        t["d_y"].copy_(0.1 * torch.randn_like(t["d_y"]))
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))
