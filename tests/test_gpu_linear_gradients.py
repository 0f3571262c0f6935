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
