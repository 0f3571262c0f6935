"""What the binding of the products, of the norms around a block and of the clipping does around a library call, on the CPU: the
library's functions are stood in for by Python functions, tensors that say they are on the GPU lie in host memory."""
import types
import weakref

import pytest
import torch


@pytest.fixture()
def stub(monkeypatch):
    import paper_2404_19760_amd as lp

    def bytes_of(*args):
        for a in args[1:]:
            if a is not None and hasattr(a, "_obj") and hasattr(a._obj, "value"):
                a._obj.value = 4096
        return lp.LP_OK

    nothing = lambda *args: lp.LP_OK  # noqa: E731
    lib = types.SimpleNamespace(lp_linear_workspace_bytes=bytes_of, lp_residual_norm_workspace_bytes=bytes_of, lp_grad_norm_workspace_bytes=bytes_of,
                                lp_linear_fwd=nothing, lp_linear_bwd=nothing, lp_residual_norm_fwd=nothing, lp_residual_norm_bwd=nothing,
                                lp_grad_norm=nothing, lp_clip_grad_norm=nothing)
    monkeypatch.setattr(lp, "_lib", lib)
    monkeypatch.setattr(lp, "_stream_ptr", lambda stream: None)
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    return lp, lib


def test_workspaces_live_through_their_calls(stub, monkeypatch):
    lp, lib = stub
    allocated, empty = [], torch.empty

    def counted(*args, **kw):
        t = empty(*args, **kw)
        if kw.get("dtype") == torch.uint8:
            allocated.append((weakref.ref(t), t.data_ptr(), t.numel()))
        return t

    seen = []

    def call(*args):
        at, size = args[-3], args[-2]
        value = lambda v: getattr(v, "value", v)  # noqa: E731
        ref, where, numel = allocated[-1]
        seen.append((ref() is not None, value(at) == where, value(size) == numel))
        return lp.LP_OK

    lib.lp_linear_bwd = lib.lp_residual_norm_bwd = lib.lp_clip_grad_norm = lib.lp_grad_norm = call
    monkeypatch.setattr(torch, "empty", counted)
    x, w = torch.zeros(10, 8), torch.zeros(4, 8)
    lp.linear_bwd(lp.Linear(w), x, None, torch.zeros(10, 4))
    lp.residual_norm_bwd(lp.ResidualNorm(), x, x.clone(), None, x)
    lp.clip_grad_norm([x], 1.0)
    lp.grad_norm([x])
    assert seen == [(True, True, True)] * 4


def test_linear_checks(stub):
    lp, lib = stub
    x, w = torch.zeros(10, 8), torch.zeros(4, 8)
    lin = lp.Linear(w)
    for bad in (torch.zeros(10, 7), torch.zeros(10, 8, dtype=torch.float64), torch.zeros(10, 8, dtype=torch.bfloat16), torch.zeros(8, 10).t()):
        with pytest.raises(ValueError):
            lp.linear_fwd(lin, bad)
    for bad in (lp.Linear(torch.zeros(8, 4).t()), lp.Linear(w, torch.zeros(5)), lp.Linear(w, torch.zeros(4, dtype=torch.bfloat16)), lp.Linear(torch.zeros(1, 4, 8)),
                lp.Linear(w, act=1 << 40)):
        with pytest.raises(ValueError):
            lp.linear_fwd(bad, x)
    for residual in (torch.zeros(10, 5), torch.zeros(9, 4), torch.zeros(10, 4, dtype=torch.float16), torch.zeros(1, 4).expand(10, 4)):
        with pytest.raises(ValueError):
            lp.linear_fwd(lin, x, residual)
    y = torch.zeros(10, 4)
    lp.lp_linear_fwd(lin, x, y, torch.zeros(10, 4), y)
    # what is written lies over something else
    wide = torch.zeros(10, 12)
    lp.lp_linear_fwd(lin, wide[:, :8], wide[:, 8:])
    with pytest.raises(ValueError, match="overlap"):
        lp.lp_linear_fwd(lin, wide[:, :8], wide[:, 7:11])
    with pytest.raises(ValueError, match="overlap"):
        lp.lp_linear_fwd(lin, wide[:, 4:], wide[:, 2:6])
    square = lp.Linear(torch.zeros(8, 8))
    for args in ((x, x), (x, x.view(-1)[:80].view(10, 8)), (x, torch.zeros(10, 8), x)):
        with pytest.raises(ValueError, match="overlap"):
            lp.lp_linear_fwd(square, *args)
    with pytest.raises(ValueError, match="overlap"):
        lp.lp_linear_fwd(lin, x, y, y)
    with pytest.raises(ValueError, match="overlap"):
        lp.lp_linear_bwd(square, x, None, torch.zeros(10, 8), x, None, None, None)
    d_y = torch.zeros(10, 8)
    with pytest.raises(ValueError, match="overlap"):
        lp.lp_linear_bwd(square, x, None, d_y, d_y, None, None, None)
    with pytest.raises(ValueError, match="strides"):
        lp.lp_linear_bwd(square, x, None, d_y, torch.zeros(10, 9)[:, :8], None, None, None)
    with pytest.raises(ValueError):
        lp.lp_linear_bwd(square, x, None, d_y, None, torch.zeros(8, 8, dtype=torch.bfloat16), None, None)
    with pytest.raises(ValueError, match="pre"):
        lp.lp_linear_bwd(square, x, torch.zeros(10, 9)[:, :8], d_y, None, None, None, None)


def test_residual_norm_checks(stub):
    lp, lib = stub
    h, f = torch.zeros(3, 5, 8), torch.zeros(3, 5, 8)
    norm = lp.ResidualNorm(gate=torch.zeros(3, 8))
    lp.residual_norm_fwd(norm, h, f)
    for bad in (lp.ResidualNorm(gate=torch.zeros(2, 8)), lp.ResidualNorm(gate=torch.zeros(3, 5, 8)), lp.ResidualNorm(gamma=torch.zeros(7)),
                lp.ResidualNorm(beta=torch.zeros(8, dtype=torch.float16)), lp.ResidualNorm(kind=1 << 33)):
        with pytest.raises(ValueError):
            lp.residual_norm_fwd(bad, h, f)
    for bad in (torch.zeros(3, 5, 7), torch.zeros(15, 8), torch.zeros(3, 5, 8, dtype=torch.float64), torch.zeros(3, 8, 5).transpose(1, 2)):
        with pytest.raises(ValueError):
            lp.residual_norm_fwd(norm, h, bad)
    with pytest.raises(ValueError, match="type of f"):
        lp.residual_norm_fwd(norm, h, f, torch.bfloat16)
    s, y = torch.zeros_like(h), torch.zeros_like(f)
    lp.lp_residual_norm_fwd(norm, h, f, h, f)
    for args in ((h, f, f, y), (h, f, s, h), (h, f, s, s)):
        with pytest.raises(ValueError, match="overlap"):
            lp.lp_residual_norm_fwd(norm, *args)
    with pytest.raises(ValueError, match="strides"):
        lp.lp_residual_norm_fwd(norm, h, f, torch.zeros(3, 5, 9)[..., :8], y)
    d_s, d_y, ws = torch.zeros_like(h), torch.zeros_like(h), torch.zeros(4096, dtype=torch.uint8)
    lp.lp_residual_norm_bwd(norm, h, f, d_s, d_y, d_s, d_y, None, None, None, None, ws)
    for d_h, d_f in ((h, None), (d_y, None), (f, None), (None, h), (None, d_s), (None, f), (d_s, d_s)):
        with pytest.raises(ValueError, match="overlap"):
            lp.lp_residual_norm_bwd(norm, h, f, d_s, d_y, d_h, d_f, None, None, None, None, ws)
    with pytest.raises(ValueError):
        lp.lp_residual_norm_bwd(norm, h, f, d_s, d_y, None, None, None, None, None, torch.zeros(8), ws)


def test_clipping_checks(stub):
    lp, lib = stub
    g = torch.zeros(4, 6)
    assert lp.clip_grad_norm([g, g.clone().t()], 1.0).shape == ()
    for bad in (torch.zeros(4, 6, dtype=torch.float64), torch.zeros(4, 6)[:, ::2], torch.zeros(1, 6).expand(4, 6)):
        with pytest.raises(ValueError):
            lp.clip_grad_norm([g, bad], 1.0)
    for outs in ([], [torch.zeros(4, 5)], [torch.zeros(6, 4).t()], [torch.zeros(4, 6, dtype=torch.float16)]):
        with pytest.raises(ValueError):
            lp.clip_grad_norm([g], 1.0, outs=outs)
    with pytest.raises(ValueError, match="no gradients"):
        lp.grad_norm([])


def test_other_devices_are_refused(stub):
    """Kernels run on the current device's stream.  (A meta tensor stands for one on another device.)"""
    lp, lib = stub
    x, w = torch.zeros(10, 8), torch.zeros(4, 8)
    there = lambda *s: torch.zeros(*s, device="meta")  # noqa: E731
    for call in (lambda: lp.linear_fwd(lp.Linear(w, there(4)), x), lambda: lp.linear_fwd(lp.Linear(w), x, there(10, 4)),
                 lambda: lp.linear_bwd(lp.Linear(w), x, None, there(10, 4)), lambda: lp.residual_norm_fwd(lp.ResidualNorm(gamma=there(8)), x),
                 lambda: lp.residual_norm_fwd(lp.ResidualNorm(), x, there(10, 8)), lambda: lp.clip_grad_norm([x, there(5)], 1.0),
                 lambda: lp.residual_norm_bwd(lp.ResidualNorm(), x, x.clone(), there(10, 8), None)):
        with pytest.raises(ValueError, match="one device"):
            call()


def test_autograd_keeps_what_may_change(stub):
    """A weight that an optimiser steps, or a sum that is written over, between forward and backward is an error."""
    lp, lib = stub
    from paper_2404_19760_amd import autograd as lpa
    x, w = torch.zeros(10, 8, requires_grad=True), torch.zeros(4, 8, requires_grad=True)
    y = lpa.linear(x, w, None, lp.LP_ACT_SILU)
    with torch.no_grad():
        w.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    f = torch.zeros(10, 8, requires_grad=True)
    s, y = lpa.residual_norm(x, f)
    with torch.no_grad():
        f.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_second_derivatives_are_an_error(stub):
    lp, lib = stub
    from paper_2404_19760_amd import autograd as lpa
    x, w = torch.randn(10, 8, requires_grad=True), torch.randn(4, 8, requires_grad=True)
    for d in torch.autograd.grad(lpa.linear(x, w, None, lp.LP_ACT_SILU).sum(), (x, w), create_graph=True):
        with pytest.raises(RuntimeError, match="first derivatives"):
            (d.square().sum() + x.square().sum()).backward()
    f = torch.randn(10, 8, requires_grad=True)
    for d in torch.autograd.grad(lpa.residual_norm(x, f)[1].sum(), (x, f), create_graph=True):
        with pytest.raises(RuntimeError, match="first derivatives"):
            (d.square().sum() + x.square().sum()).backward()


def test_clipping_of_parameters(stub):
    lp, lib = stub
    from paper_2404_19760_amd.optim import clip_grad_norm_
    calls = []
    lib.lp_clip_grad_norm = lambda *args: calls.append(args[0]) or lp.LP_OK
    params = [torch.zeros(3, requires_grad=True) for _ in range(4)]
    assert float(clip_grad_norm_(params, 1.0)) == 0.0 and not calls
    for p in params[:3]:
        p.grad = torch.ones(3)
    clip_grad_norm_([*params, params[0]], 1.0)   # (one listed twice is scaled once)
    clip_grad_norm_(params[0], 1.0)
    assert calls == [3, 1]
