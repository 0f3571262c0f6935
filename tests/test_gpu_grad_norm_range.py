"""Clipping where the factor is no normal number of fp32: results that are must come out as exactly as others.

A factor in fp64 is good to some 2^-52; its product with a value is rounded to fp32 (u = 2^-24, or half of fp32's smallest number) and to the
tensor's type (half a step, or half of its smallest number)."""
import math

import pytest
import torch

from test_gpu_grad_norm import SMALLEST, U, _norm, _tensors

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("sizes", [[100], [7, 1023, 30000], [50003], [50003, 3, 70001], [4097] * 70])
@pytest.mark.parametrize("max_norm", [1e-3, 1e-6, 1e-30, 1e-39])
def test_largest_gradients_under_a_small_norm(lp, sizes, dtype, max_norm):
    for shift in (0, 1):
        grads = _tensors(sizes, dtype, len(sizes), scale=1e36, shift=shift)
        want = _norm(grads)
        factor = torch.tensor(max_norm).item() / want
        assert factor < 2.0 ** -126
        outs = [torch.full_like(g, 9.0) for g in grads]
        norm = lp.clip_grad_norm(grads, max_norm, 0.0, outs)
        assert abs(float(norm) - want) <= 1.01 * U * want if want < 3e38 else float(norm) > 2.9e38
        lp.clip_grad_norm(grads_too := [g.clone() for g in grads], max_norm, 0.0)
        for g, o, p in zip(grads, outs, grads_too):
            exact = g.double() * factor
            bound = (1.01 * U + (0 if dtype == torch.float32 else torch.finfo(dtype).eps / 2)) * exact.abs() + 0.51 * (2.0 ** -149 + SMALLEST[dtype])
            assert bool(((o.double() - exact).abs() <= 1.01 * bound).all())
            assert torch.equal(o, p)
        assert max_norm < 1e-38 or math.sqrt(math.fsum(float(o.double().square().sum()) for o in outs)) > 0.99 * torch.tensor(max_norm).item()


@pytest.mark.parametrize("sizes", [[100], [50003, 3]])
def test_a_largest_norm_of_zero(lp, sizes):
    grads = _tensors(sizes, torch.float32, 3)
    lp.clip_grad_norm(grads, 0.0)
    assert not any(g.any() for g in grads)


@pytest.mark.parametrize("sizes", [[100], [50003, 3]])
def test_norms_beyond_fp32(lp, sizes):
    """The norm is given as infinite; the gradients, all of them finite, still come under the largest norm."""
    grads = [torch.full((s,), 3e38, device="cuda") for s in sizes]
    total = sum(sizes)
    assert math.isinf(float(lp.clip_grad_norm(grads, 5.0)))
    for g in grads:
        assert float((g.double() * math.sqrt(total) / 5.0 - 1).abs().max()) <= 3 * U
