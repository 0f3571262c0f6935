"""The norm of all gradients together, and clipping, against 64 bits.

The sum of squares is fp64, so the norm is off by its rounding to fp32 (2^-24) and some 2^-50; the factor is rounded to fp32 and the product
with a value once more in fp32 (2^-24 each), then the result to its type by half a step (16-bit types: never more than half of their
smallest number)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SMALLEST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}
LISTS = [[1], [5], [4, 4], [3, 1, 2, 7, 8, 9, 15, 16], [1023, 1025], [32768], [32769], [8191, 8193, 4, 3], [100000], [1, 200001, 7], [7] * 9,
         [5, 4096, 4097, 12288, 1] * 30, [3000001, 1, 999], [513] * 700, [17] * 5000]


def _tensors(sizes, dtype, seed, scale=1.0, shift=0):
    """Tensors of these sizes, each `shift` elements behind the start of its allocation."""
    gen = torch.Generator().manual_seed(seed)
    return [(scale * 10.0 ** (k % 3 - 1) * torch.randn(s + shift, generator=gen)).to(dtype).cuda()[shift:] for k, s in enumerate(sizes)]


def _norm(grads):
    return math.sqrt(math.fsum(float(g.double().cpu().square().sum()) for g in grads))


def _check(grads, outs, norm, max_norm, eps):
    want = _norm(grads)
    assert abs(float(norm) - want) <= 1.01 * U * want
    factor = min(1.0, max_norm / (want + eps)) if want else 1.0
    for g, o in zip(grads, outs):
        exact = g.double() * factor
        bound = (2.01 * U * (factor < 1) + torch.finfo(g.dtype).eps / 2 * (factor < 1 and g.dtype != torch.float32)) * exact.abs() + 0.51 * SMALLEST[g.dtype]
        assert bool(((o.double() - exact).abs() <= 1.01 * bound).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("sizes", LISTS, ids=lambda s: f"{len(s)}x{s[0]}")
def test_norm_and_clipping(lp, sizes, dtype):
    for shift, part in ((0, 0.3), (1, 0.5), (3, 2.0), (0, 1e-3)):
        grads = _tensors(sizes, dtype, len(sizes) + shift, shift=shift)
        want = _norm(grads)
        got = lp.grad_norm(grads)
        assert got.shape == () and abs(float(got) - want) <= 1.01 * U * want
        outs = [torch.full_like(g, 9.0) for g in grads]   # (aligned otherwise than the gradients)
        kept = [g.clone() for g in grads]
        norm = lp.clip_grad_norm(grads, part * want, outs=outs)
        assert torch.equal(norm, got) and all(torch.equal(a, b) for a, b in zip(grads, kept))
        _check(grads, outs, norm, torch.tensor(part * want).item(), 1e-6)
        norm = lp.clip_grad_norm(grads, part * want)
        assert torch.equal(norm, got) and all(torch.equal(a, b) for a, b in zip(grads, outs))


def test_mixed_types_and_empty_tensors(lp):
    grads = [t for d, s in ((torch.float32, [5, 0, 70000]), (torch.bfloat16, [33, 4097]), (torch.float16, [0, 1, 9000])) for t in _tensors(s, d, 3)]
    kept = [g.clone() for g in grads]
    norm = lp.clip_grad_norm(grads, 1.0)
    _check(kept, grads, norm, 1.0, 1e-6)
    assert float(lp.grad_norm([torch.empty(0, device="cuda")])) == 0.0
    zeros = [torch.zeros(100, device="cuda"), torch.zeros(50000, device="cuda")]
    for few in (zeros[:1], zeros):
        for eps in (0.0, 1e-6):
            assert float(lp.clip_grad_norm(few, 0.0, eps)) == 0.0 and not any(z.any() for z in few)


def test_values_beside_the_tensors_stay(lp):
    for size in (1001, 70001):
        wide = torch.full((size + 14,), 5.0, device="cuda")
        grad = wide[7:7 + size]
        grad.normal_()
        lp.clip_grad_norm([grad], 0.1)
        assert bool((wide[:7] == 5.0).all()) and bool((wide[7 + size:] == 5.0).all())
        assert abs(float(grad.double().norm()) - 0.1) < 1e-6


@pytest.mark.parametrize("sizes", [[100], [50000, 3]])
def test_values_whose_squares_do_not_fit_fp32(lp, sizes):
    """3e38 and 1e-40: squares beyond and below fp32."""
    for scale in (1e37, 1e-30):
        grads = [torch.full((s,), scale, device="cuda") for s in sizes]
        want = float(torch.tensor(scale)) * math.sqrt(sum(sizes))
        norm = lp.grad_norm(grads)
        assert math.isinf(float(norm)) if want > 3.4028235e38 else abs(float(norm) - want) <= 2 * U * want
        norm = lp.clip_grad_norm(grads, want / 2 if want < 3e38 else 1e38, 0.0)
        if want < 3e38:
            assert abs(float(grads[0].double()[0]) / float(torch.tensor(scale).double()) - 0.5) < 1e-6


@pytest.mark.parametrize("sizes", [[100, 7], [50000, 3]])
def test_norms_that_are_not_finite(lp, sizes):
    grads = _tensors(sizes, torch.float32, 1)
    grads[0][3] = float("inf")
    assert math.isinf(float(lp.clip_grad_norm(grads, 1.0)))
    assert bool(torch.isnan(grads[0][3])) and not grads[0][:3].any() and not grads[1].any()
    grads = _tensors(sizes, torch.float32, 1)
    grads[1][0] = float("nan")
    assert math.isnan(float(lp.clip_grad_norm(grads, 1.0)))
    assert all(torch.isnan(g).all() for g in grads)


def test_gradients_in_other_orders_and_versions(lp):
    gen = torch.Generator().manual_seed(2)
    a = torch.randn(40, 50, generator=gen).cuda().t()
    b = torch.randn(300, 200, generator=gen).cuda().t()
    for grads in ([a.clone().t().contiguous().t()], [a.contiguous().t().contiguous().t(), b.contiguous().t().contiguous().t()]):
        kept, version = [g.clone() for g in grads], grads[0]._version
        norm = lp.clip_grad_norm(grads, 2.0)
        _check(kept, grads, norm, 2.0, 1e-6)
        assert grads[0]._version > version
    with pytest.raises(ValueError, match="dense"):
        lp.clip_grad_norm([torch.zeros(10, 10, device="cuda")[:, :5]], 1.0)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_more_than_the_cache_holds(lp, dtype):
    """Results of such calls are stored another way; at odd addresses."""
    size = 300_000_000 // torch.finfo(dtype).bits * 8
    wide = torch.randn(size + 9, device="cuda").to(dtype)
    grads = [wide[3:3 + size], torch.randn(1001, device="cuda").to(dtype)]
    want = [g.float().clone() for g in grads]
    edges = wide[:3].clone(), wide[3 + size:].clone()
    norm = lp.clip_grad_norm(grads, 7.0, 0.0)
    exact = math.sqrt(sum(float(torch.linalg.vector_norm(g, dtype=torch.float64)) ** 2 for g in want))
    assert abs(float(norm) - exact) <= 1.01 * U * exact
    factor = torch.tensor(7.0 / exact, dtype=torch.float64).float().cuda()   # (as the library rounds it, but for the norm's last bits)
    for g, w in zip(grads, want):
        assert bool(((g.float() - w * factor).abs() <= (4 * U + torch.finfo(dtype).eps * (dtype != torch.float32)) * (w * factor).abs() + SMALLEST[dtype]).all())
    assert torch.equal(wide[:3], edges[0]) and torch.equal(wide[3 + size:], edges[1])


def test_captured_and_replayed(lp):
    for sizes in ([64 * 16, 64, 64 * 64], [100000, 7, 30000] * 30):
        grads = _tensors(sizes, torch.float32, 9)
        outs = [torch.empty_like(g) for g in grads]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            lp.clip_grad_norm(grads, 1.0, outs=outs)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = lp.clip_grad_norm(grads, 1.0, outs=outs)
        for _ in range(4):
            for g in grads:
                g.normal_()
            graph.replay()
            got = [held.clone(), *[o.clone() for o in outs]]
            want = [lp.clip_grad_norm(grads, 1.0, outs=outs), *outs]
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(got, want))
