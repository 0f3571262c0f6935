"""Gradients of products where some of them are not wanted, and calls that tests of all gradients together do not make."""
import ctypes as C

import pytest
import torch

from test_gpu_linear import DTYPES, _act_id, _case, _check_backward

pytestmark = pytest.mark.gpu


def _pre(t, act, dtype):
    return None if act == "none" else (t["x"].double().cpu() @ t["w"].double().cpu().T + t["b"].double().cpu()).to(dtype).cuda()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("p,k,n", [(700, 32, 64), (700, 33, 97), (700, 5, 3), (65, 128, 128), (700, 33, 140), (700, 136, 200), (7, 64, 24)])
def test_gradients_that_do_not_need_x(lp, p, k, n, dtype):
    """x is read for the weight's gradient alone: without it a call may pass NULL, and its results are those of a call for all gradients."""
    for act in ("none", "silu"):
        t = _case(p, k, n, dtype, p + k + n, "odd")
        pre = _pre(t, act, dtype)
        lin = lp.Linear(t["w"], t["b"], _act_id(lp, act))
        whole = lp.linear_bwd(lin, t["x"], pre, t["d_y"])
        _check_backward(t, act, dtype, pre, *whole)
        q = lin.c_struct(t["x"], t["d_y"].stride(0))
        size = lp.lp_linear_workspace_bytes(lin, t["x"])[1]
        ws = torch.empty(size, dtype=torch.uint8, device="cuda")
        at = lambda v: None if v is None else v.data_ptr()  # noqa: E731
        for wanted in range(1, 4):
            for x in (t["x"], None):
                d_x = torch.empty_strided(t["x"].shape, t["x"].stride(), dtype=dtype, device="cuda") if wanted & 1 else None
                d_b = torch.zeros(n, device="cuda") if wanted & 2 else None
                assert lp._lib.lp_linear_bwd(C.byref(q), at(x), at(pre), t["d_y"].data_ptr(), at(d_x), None, at(d_b), at(ws), size,
                                             torch.cuda.current_stream().cuda_stream) == lp.LP_OK
                assert d_b is None or torch.equal(d_b, whole[2])
                if d_x is None:
                    continue
                # (d_x of more than 128 channels comes from another kernel where d_z was not made for d_bias)
                if k > 128:
                    _check_backward(t, act, dtype, pre, d_x, whole[1], whole[2])
                else:
                    assert torch.equal(d_x, whole[0])


# channels in and out: every tile of the gradients' kernel, rows that end with whole chunks and others
TILES = [(32, 64), (64, 64), (128, 64), (32, 128), (64, 128), (128, 128), (31, 61), (61, 33), (125, 97), (5, 3), (72, 200), (200, 136), (512, 160),
         (129, 145), (515, 131)]
MANY = [(65537 + 14, *t) for t in TILES] + [(p, *t) for p in (65535, 65536, 150001) for t in ((32, 128), (33, 97), (72, 200))] + [(4099, *t) for t in TILES[:9]]


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("p,k,n", MANY)
def test_weight_gradients_hold_all_bits_of_d_z(lp, p, k, n, dtype, act):
    """Every channel of d_y is zero but in one position, so d_bias is that position's d_z as the kernel has it in fp32, and d_weight is d_z times
    that position's x, without sums that could hide what d_z was rounded to on the way.  With u = 2^-24: three bf16 parts leave (2^-8)^3 = u of
    d_z and their products are exact, two u for each of the three additions; fp16 and bf16 parts leave 2^-11 2^-8, x is rounded to bf16 for
    the second part, 2^-11 2^-8 again (the first part of a d_z among fp16's smallest numbers is off by up to 2^-25); fp32 products and additions are
    rounded by two u.  Largest in all: 8 u, and two times 2^-19, or 2^-33 of x, more in fp16."""
    gen = torch.Generator().manual_seed(p + k + n)
    rows = torch.arange(n) * (p - 1) // max(1, n - 1)
    x = torch.randn(p, k, generator=gen).to(dtype).cuda()
    pre = torch.randn(p, n, generator=gen).to(dtype).cuda()
    d_y = torch.zeros(p, n, dtype=dtype, device="cuda")
    d_y[rows.cuda(), torch.arange(n, device="cuda")] = (1 + torch.rand(n, generator=gen)).to(dtype).cuda()
    w = torch.randn(n, k, generator=gen).to(dtype).cuda()
    _, d_w, d_b = lp.linear_bwd(lp.Linear(w, torch.zeros(n, device="cuda"), _act_id(lp, act)), x, pre, d_y)
    assert rows[-1] == p - 1 and (n == 1 or bool((d_b != 0).all()))
    want = d_b.double().unsqueeze(1) * x[rows.cuda()].double()
    bound = 8 * 2.0 ** -24 * want.abs()
    if dtype == torch.float16:
        bound = bound + 2.01 * (2.0 ** -19 * want.abs() + 2.0 ** -33 * x[rows.cuda()].double().abs())
    over = ((d_w.double() - want).abs() - bound).max()
    assert float(over) <= 0, float(((d_w.double() - want).abs() / want.abs()).max())


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("p,k,n", [(65535, 32, 128), (65536, 32, 128), (65537, 33, 97), (65551, 72, 200), (65536, 136, 160)])
def test_gradients_of_many_positions(lp, p, k, n, act):
    t = _case(p, k, n, torch.bfloat16, p, "odd" if p % 2 else "")
    pre = _pre(t, act, torch.bfloat16)
    d_x, d_w, d_b = lp.linear_bwd(lp.Linear(t["w"], t["b"], _act_id(lp, act)), t["x"], pre, t["d_y"])
    _check_backward(t, act, torch.bfloat16, pre, d_x, d_w, d_b)


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu"])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("p,k,n", [(700, 136, 200), (513, 264, 130), (30, 200, 72), (1000, 145, 257)])
def test_gradients_through_frozen_weights(lp, p, k, n, dtype, act):
    """x alone wants a gradient: more than 128 channels of it, which come straight from d_y and pre, through autograd and the entry point."""
    from paper_2404_19760_amd import autograd as lpa
    t = _case(p, k, n, dtype, p + k + n, "odd")
    x = t["x"].detach().requires_grad_(True)
    lpa.linear(x, t["w"], t["b"], _act_id(lp, act)).backward(t["d_y"])
    lin = lp.Linear(t["w"], t["b"], _act_id(lp, act))
    _, pre = lp.linear_fwd(lin, t["x"], keep=True)
    pre = None if act == "none" else pre
    ws = torch.empty(lp.lp_linear_workspace_bytes(lin, t["x"])[1], dtype=torch.uint8, device="cuda")
    d_x = torch.empty_strided(t["x"].shape, t["x"].stride(), dtype=dtype, device="cuda")
    lp.lp_linear_bwd(lin, t["x"], pre, t["d_y"], d_x, None, None, ws)
    _, d_w, d_b = lp.linear_bwd(lin, t["x"], pre, t["d_y"])
    _check_backward(t, act, dtype, pre, d_x, d_w, d_b)
    assert torch.equal(x.grad, d_x)
