"""What the binding of the norm and of the orthogonalised updates does around a library call, on the CPU: the library's functions are
stood in for by Python functions, tensors that say they are on the GPU lie in host memory."""
import types
import weakref

import pytest
import torch


@pytest.fixture()
def stub(monkeypatch):
    """The binding with a library whose calls do nothing but what a test puts in their place."""
    import paper_2404_19760_amd as lp

    def bytes_of_norm(norm, fwd, bwd):
        fwd._obj.value, bwd._obj.value = 4096, 8192
        return lp.LP_OK

    lib = types.SimpleNamespace(lp_group_norm_workspace_bytes=bytes_of_norm)
    monkeypatch.setattr(lp, "_lib", lib)
    monkeypatch.setattr(lp, "_stream_ptr", lambda stream: None)
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    return lp, lib


def test_workspace_of_the_norm_lives_through_the_call(stub, monkeypatch):
    """The kernels are enqueued inside the call: until it returns nobody else may be given the memory (the call gives up the
    interpreter's lock, so other threads allocate meanwhile)."""
    lp, lib = stub
    allocated, empty = [], torch.empty

    def counted(*args, **kw):
        t = empty(*args, **kw)
        if kw.get("dtype") == torch.uint8:
            allocated.append((weakref.ref(t), t.data_ptr(), t.numel()))
        return t

    seen = []

    def call(*args):
        workspace, size = args[-3], args[-2]
        ref, at, numel = allocated[-1]
        seen.append((ref() is not None, workspace == at, size == numel))
        return lp.LP_OK

    lib.lp_group_norm_fwd = lib.lp_group_norm_bwd = call
    monkeypatch.setattr(torch, "empty", counted)
    x = torch.zeros(2, 10, 8)
    _, stats = lp.group_norm_fwd(lp.GroupNorm(2), x)
    lp.group_norm_bwd(lp.GroupNorm(2), x, torch.zeros(2, 2, 2), x)
    assert seen == [(True, True, True)] * 2


def _norm_calls_do_nothing(lp, lib):
    lib.lp_group_norm_fwd = lib.lp_group_norm_bwd = lambda *args: lp.LP_OK


def test_occupancy_that_changes_before_the_backward_is_an_error(stub):
    """A weight buffer that is splatted into again between forward and backward: the gradients would be those of another norm."""
    lp, lib = stub
    from paper_2404_19760_amd import autograd as lpa
    _norm_calls_do_nothing(lp, lib)
    x = torch.randn(1, 10, 8, requires_grad=True)
    occupancy = torch.ones(1, 10)
    y = lpa.group_norm(x, 2, occupancy=occupancy)
    y.sum().backward()
    y = lpa.group_norm(x, 2, occupancy=occupancy)
    occupancy.zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_second_derivatives_of_the_norm_are_an_error(stub):
    """The backward's kernels are not differentiable: where another path exists, a gradient penalty would lose its term without a word."""
    lp, lib = stub
    from paper_2404_19760_amd import autograd as lpa
    _norm_calls_do_nothing(lp, lib)
    x, gamma = torch.randn(1, 10, 8, requires_grad=True), torch.ones(8, requires_grad=True)
    y = lpa.group_norm(x, 2, gamma)
    d_x, d_gamma = torch.autograd.grad(y.sum(), (x, gamma), create_graph=True)
    for d in (d_x, d_gamma):
        with pytest.raises(RuntimeError, match="first derivatives"):
            (d.square().sum() + x.square().sum()).backward()


def test_second_derivatives_of_the_renderer_are_an_error(stub):
    """The same of the Renderer, for its grid, weights and biases."""
    lp, lib = stub
    from paper_2404_19760_amd import autograd as lpa

    def bytes_of_backward(*args):
        args[-1]._obj.value = 4096
        return lp.LP_OK

    lib.lp_bwd_workspace_bytes = bytes_of_backward
    lib.lp_render_fwd = lib.lp_render_bwd = lambda *args: lp.LP_OK
    data = torch.randn(1, 4, 4, 4, 16, requires_grad=True)
    weights = [torch.randn(*s, requires_grad=True) for s in ((32, 16), (4, 32))]
    biases = [torch.randn(s, requires_grad=True) for s in (32, 4)]
    one = torch.ones(5)
    rays = lp.Rays(torch.zeros(5, 3), torch.ones(5, 3), one, 2 * one, 8)
    rgb, alpha, depth = lpa.render(lp.Grid(lp.LP_GRID_VOXEL, [data], (4, 4, 4)), lp.Mlp(weights, biases), rays, (0.0, 0.0, 0.0))
    inputs = [data, *weights, *biases]
    grads = torch.autograd.grad(rgb.sum() + alpha.sum(), inputs, create_graph=True)
    for d in grads:
        with pytest.raises(RuntimeError, match="first derivatives"):
            (d.square().sum() + sum(t.square().sum() for t in inputs)).backward(retain_graph=True)
    for t in inputs:
        t.grad = None
    (rgb.sum() + depth.sum()).backward()
    assert all(t.grad is not None for t in inputs)


def test_what_a_call_writes_counts_as_written(stub):
    """Tensors written through their addresses move in their version, so that a graph that has saved them notices."""
    lp, lib = stub
    _norm_calls_do_nothing(lp, lib)
    lib.lp_muon_step = lib.lp_orthogonalize = lambda *args: lp.LP_OK

    def moved(call, written, read):
        before = [t._version for t in (*written, *read)]
        call()
        after = [t._version for t in (*written, *read)]
        assert after == [b + (k < len(written)) for k, b in enumerate(before)]

    w, g, m = ([torch.zeros(4, 4) for _ in range(2)] for _ in range(3))
    ws = torch.zeros(16, dtype=torch.uint8)
    moved(lambda: lp.lp_muon_step([t.detach() for t in w], g, m, ws, lr=0.1), w + m, g)
    moved(lambda: lp.lp_orthogonalize(g, m, ws), m, g)
    moved(lambda: lp.lp_orthogonalize(g, g, ws), g, m)
    x, y, d_x, stats, gamma, beta = torch.zeros(2, 10, 8), torch.zeros(2, 10, 8), torch.zeros(2, 10, 8), torch.zeros(2, 2, 2), torch.zeros(8), torch.zeros(8)
    norm = lp.GroupNorm(2)
    moved(lambda: lp.lp_group_norm_fwd(norm, x, y, stats, None), [y, stats], [x])
    moved(lambda: lp.lp_group_norm_fwd(norm, x, x, None, None), [x], [])
    moved(lambda: lp.lp_group_norm_bwd(norm, x, stats, y, d_x, gamma, beta, None), [d_x, gamma, beta], [x, stats, y])
    moved(lambda: lp.lp_group_norm_bwd(norm, x, stats, y, None, None, beta, None), [beta], [x, stats, y])
    with torch.inference_mode():   # (tensors without a version)
        w, g, m = ([torch.zeros(4, 4)] for _ in range(3))
    lp.lp_muon_step(w, g, m, ws, lr=0.1)


def test_a_graph_notices_a_step_of_the_optimiser(stub):
    """The backward of a graph that was kept over the step would use the new weights as if they were the old ones."""
    lp, lib = stub
    from paper_2404_19760_amd.optim import Muon

    def bytes_of_step(n, lists, size):
        size._obj.value = 256
        return lp.LP_OK

    lib.lp_muon_workspace_bytes, lib.lp_muon_step = bytes_of_step, lambda *args: lp.LP_OK
    w = torch.randn(4, 4, requires_grad=True)
    x = torch.randn(3, 4, requires_grad=True)
    loss = (x @ w).square().sum()
    loss.backward(retain_graph=True)
    Muon([w]).step()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()


def test_overlap_of_what_is_written_and_what_is_read(stub):
    """Slices of one tensor that share channels are refused (some threads would read what others have written), slices side by side,
    tensors behind one another and a tensor itself are taken."""
    lp, lib = stub
    _norm_calls_do_nothing(lp, lib)
    norm = lp.GroupNorm(2)
    wide = torch.zeros(2, 5, 3, 24)
    flat = torch.zeros(2 * 5 * 3 * 24)
    halves = wide.view(torch.bfloat16)   # [..., 48], bytes as in `wide`
    at = lambda a, c: wide[..., a:a + c]  # noqa: E731
    lone = torch.zeros(1, 1, 8, 16)
    taken = [(at(0, 8), at(8, 8)), (at(8, 8), at(0, 8)), (at(0, 12), at(12, 12)), (at(4, 8), at(4, 8)), (wide[:1], wide[1:]), (at(0, 8)[:1], at(4, 8)[1:]),
             (at(4, 8)[1:], at(0, 8)[:1]), (flat[:80].view(1, 10, 8), flat[80:160].view(1, 10, 8)), (at(0, 8), halves[..., 16:24]),
             (lone[:, 0], lone[:, 0].as_strided((1, 8, 16), (7, 16, 1)))]
    refused = [(at(0, 8), at(4, 8)), (at(4, 8), at(0, 8)), (at(0, 8), at(7, 8)), (at(7, 8), at(0, 8)), (at(0, 8)[:1], at(1, 8)[:1]),
               (at(0, 8)[:1, 1:], at(4, 8)[:1, :-1]), (at(0, 8), halves[..., 14:22]),
               (at(0, 8), halves[..., 0:8]), (flat[:80].view(1, 10, 8), flat[79:159].view(1, 10, 8)), (flat[8:88].view(1, 10, 8), flat[:80].view(1, 10, 8)),
               (wide, wide.view(torch.bfloat16)[..., :24]), (flat[:80].view(1, 10, 8), flat[:160].view(1, 10, 16)[..., 8:])]
    for x, y in taken:
        lp.lp_group_norm_fwd(norm, x, y, None, None)
    for x, y in refused:
        with pytest.raises(ValueError, match="overlap"):
            lp.lp_group_norm_fwd(norm, x, y, None, None)
    x, stats = torch.zeros(2, 5, 3, 24)[..., :8], torch.zeros(2, 2, 2)
    lp.lp_group_norm_bwd(norm, x, stats, at(0, 8), at(0, 8), None, None, None)
    lp.lp_group_norm_bwd(norm, x, stats, at(0, 8), at(8, 8), None, None, None)
    with pytest.raises(ValueError, match="overlap"):
        lp.lp_group_norm_bwd(norm, x, stats, at(0, 8), at(4, 8), None, None, None)
    with pytest.raises(ValueError, match="overlap"):
        lp.lp_group_norm_bwd(norm, at(0, 8), stats, x, at(4, 8), None, None, None)


def test_groups_added_to_the_optimiser_are_checked(stub):
    """As those given to the constructor: a vector or a 16-bit matrix would end a later step, behind groups that were stepped already."""
    from paper_2404_19760_amd.optim import Muon
    opt = Muon([torch.zeros(4, 4)])
    for bad in ([torch.zeros(8)], [torch.zeros(4, 4), torch.zeros(4, 4, dtype=torch.float16)], torch.zeros(8)):
        with pytest.raises(ValueError, match="matrices"):
            opt.add_param_group({"params": bad})
        assert len(opt.param_groups) == 1
    opt.add_param_group({"params": [torch.zeros(2, 3, 4)], "lr": 0.5})
    assert [g["lr"] for g in opt.param_groups] == [0.02, 0.5]
    with pytest.raises(ValueError, match="matrices"):
        Muon([{"params": [torch.zeros(4, 4)]}, {"params": [torch.zeros(8)]}])


def test_coefficients_without_any_are_refused(stub):
    lp, _ = stub
    for empty in ((), []):
        with pytest.raises(ValueError, match="every step"):
            lp._orth(5, empty, 0.0)


def test_numbers_beyond_32_bits_are_refused(stub):
    """The C structs hold 32 bits of them; what is beyond would be cut off without a word (2^32 + 8 columns taken for 8)."""
    lp, lib = stub
    _norm_calls_do_nothing(lp, lib)
    lib.lp_orthogonalize = lib.lp_muon_step = lambda *args: lp.LP_OK
    meta = lambda *shape: torch.empty(shape, device="meta")  # noqa: E731
    ws, small = torch.zeros(16, dtype=torch.uint8), meta(4, 4)
    for big in (meta(2, 2 ** 32 + 8), meta(2 ** 32 + 8, 2), meta(2, 2 ** 31)):
        with pytest.raises(ValueError, match="32 bits"):
            lp.lp_orthogonalize([big], [big], ws)
        with pytest.raises(ValueError, match="32 bits"):
            lp.lp_muon_step([big], [big], [big], ws, lr=0.1)
    for kw in (dict(steps=2 ** 32 + 5), dict(steps=2 ** 32 + 5, coeffs=(1.0, 0.0, 0.0)), dict(steps=-2 ** 40)):
        with pytest.raises(ValueError, match="32 bits"):
            lp.lp_orthogonalize([small], [small], ws, **kw)
    for kw in (dict(scale=2 ** 32), dict(nesterov=2 ** 32 + 1)):
        with pytest.raises(ValueError, match="32 bits"):
            lp.lp_muon_step([small], [small], [small], ws, lr=0.1, **kw)
    x = meta(1, 3, 2 ** 32 + 8)
    with pytest.raises(ValueError, match="32 bits"):
        lp.lp_group_norm_fwd(lp.GroupNorm(2), x, torch.empty_like(x), None, None)
    x = meta(1, 3, 8)
    for norm in (lp.GroupNorm(2 ** 32 + 2), lp.GroupNorm(2, act=2 ** 32 + lp.LP_ACT_SILU)):
        with pytest.raises(ValueError, match="32 bits"):
            lp.lp_group_norm_fwd(norm, x, torch.empty_like(x), None, None)
