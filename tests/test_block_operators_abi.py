"""Argument errors of the products, of the norms around a block and of the clipping are statuses before anything touches a GPU.  CPU only."""
import ctypes as C

import pytest


@pytest.fixture()
def lp():
    import paper_2404_19760_amd as lp
    return lp


def _set(q, kw):
    for k, v in kw.items():
        setattr(q, k, v)
    return q


def test_gradients_are_packed_as_they_are_laid_out(lp):
    """The binding makes the structs of a list of gradients from one buffer."""
    import struct
    assert struct.calcsize("qQQi4x") == C.sizeof(lp._Gradient)
    q = lp._Gradient.from_buffer(bytearray(struct.pack("qQQi4x", 1, 2, 3, 4)))
    assert (q.size, q.input, q.out, q.dtype) == (1, 2, 3, 4)


def test_linear_refusals(lp):
    lib = lp._lib
    one = C.c_void_p(4096)

    def q(**kw):
        return _set(lp._Linear(10, 8, 8, lp.LP_ACT_SILU, lp.LP_F32, 0, 0, 0, 4096, None, None), kw)

    def fwd(l, x=one, y=one):
        return lib.lp_linear_fwd(l and C.byref(l), x, y, None, None, 0, None)

    def bwd(l, x=one, pre=one, dy=one, dx=one, dw=one):
        return lib.lp_linear_bwd(l and C.byref(l), x, pre, dy, dx, dw, None, None, 0, None)

    for call in (fwd, bwd):
        assert call(None) == lp.LP_ERR_INVALID_ARG and b"NULL" in lib.lp_last_error()
        for kw, word in ((dict(P=-1), b"P"), (dict(K=0), b"K"), (dict(N=0), b"N"), (dict(N=-5), b"N"), (dict(act=4), b"act"), (dict(act=-1), b"act"),
                         (dict(dtype=3), b"dtype"), (dict(x_stride=7), b"stride"), (dict(y_stride=-8), b"stride"), (dict(r_stride=3), b"stride"),
                         (dict(weight=None), b"weight"), (dict(weight=4098), b"aligned")):
            assert call(q(**kw)) == lp.LP_ERR_INVALID_ARG and word in lib.lp_last_error(), kw
        assert call(q(K=(1 << 20) + 1)) == lp.LP_ERR_UNSUPPORTED and call(q(N=1 << 30)) == lp.LP_ERR_UNSUPPORTED
        assert call(q(P=1 << 60)) == lp.LP_ERR_UNSUPPORTED
        assert call(q(P=0)) == lp.LP_OK   # nothing to do
    assert fwd(q(), x=None) == fwd(q(), y=None) == fwd(q(), x=C.c_void_p(4097)) == lp.LP_ERR_INVALID_ARG
    assert bwd(q(), dy=None) == bwd(q(), pre=None) == bwd(q(), x=None) == lp.LP_ERR_INVALID_ARG
    n = C.c_size_t(7)
    assert lib.lp_linear_workspace_bytes(C.byref(q(act=7)), C.byref(n), None) == lp.LP_ERR_INVALID_ARG


def test_residual_norm_refusals(lp):
    lib = lp._lib
    one = C.c_void_p(4096)

    def q(**kw):
        return _set(lp._ResidualNorm(2, 10, 8, lp.LP_NORM_RMS, 0, 0, 1.0, 1e-5, lp.LP_F32, lp.LP_F32, 0, 0, 0, None, None, None, None), kw)

    def fwd(l, h=one):
        return lib.lp_residual_norm_fwd(l and C.byref(l), h, one, one, one, None)

    def bwd(l, h=one, f=one, d_f=one, d_post=None, d_gate=None):
        return lib.lp_residual_norm_bwd(l and C.byref(l), h, f, one, one, one, d_f, None, None, d_post, d_gate, None, 0, None)

    for call in (fwd, bwd):
        assert call(None) == lp.LP_ERR_INVALID_ARG and b"NULL" in lib.lp_last_error()
        for kw, word in ((dict(N=-1), b"N"), (dict(P=-1), b"P"), (dict(C=0), b"C"), (dict(kind=2), b"kind"), (dict(post_norm=2), b"0 or 1"),
                         (dict(gate_per_sample=-1), b"0 or 1"), (dict(eps=-1.0), b"eps"), (dict(eps=float("nan")), b"eps"),
                         (dict(alpha=float("inf")), b"alpha"), (dict(h_dtype=3), b"dtype"), (dict(f_dtype=-1), b"dtype"), (dict(h_stride=7), b"stride"),
                         (dict(f_stride=-1), b"stride"), (dict(y_stride=2), b"stride"), (dict(post_gamma=4096), b"post_norm")):
            assert call(q(**kw)) == lp.LP_ERR_INVALID_ARG and word in lib.lp_last_error(), kw
        assert call(q(C=8193)) == call(q(h_dtype=lp.LP_BF16)) == call(q(N=1 << 40, P=1 << 40)) == lp.LP_ERR_UNSUPPORTED
        assert call(q(N=0)) == call(q(P=0)) == lp.LP_OK   # nothing to do
        assert call(q(), h=None) == call(q(), h=C.c_void_p(4098)) == lp.LP_ERR_INVALID_ARG
    assert bwd(q(), f=None) == bwd(q(), f=None, d_f=None, d_gate=one) == bwd(q(), d_post=one) == lp.LP_ERR_INVALID_ARG


def test_clipping_refusals(lp):
    lib = lp._lib
    norm = C.c_void_p(1 << 20)

    def clip(lists, max_norm=1.0, eps=1e-6, norm=norm, n=None):
        arr = (lp._Gradient * max(1, len(lists)))(*[lp._Gradient(*g) for g in lists])
        return lib.lp_clip_grad_norm(len(lists) if n is None else n, arr, max_norm, eps, norm, None, 0, None)

    a, b, c = 4096, 8192, 16384
    good = (64, a, b, lp.LP_F32)
    for lists, word in (([(64, a, b, 3)], b"dtype"), ([(-1, a, b, 0)], b"size"), ([(64, None, b, 0)], b"NULL"), ([(64, a, None, 0)], b"NULL"),
                        ([(64, a + 2, b, 0)], b"aligned"), ([(64, a, b + 1, lp.LP_BF16)], b"aligned"), ([good, (64, a, b, 7)], b"grads[1]")):
        assert clip(lists) == lp.LP_ERR_INVALID_ARG and word in lib.lp_last_error(), lists
    for kw in (dict(max_norm=-1.0), dict(max_norm=float("inf")), dict(max_norm=float("nan")), dict(eps=-1.0), dict(eps=float("inf")),
               dict(norm=None), dict(n=-1)):
        assert clip([good], **kw) == lp.LP_ERR_INVALID_ARG, kw
    # what is written lies over something else
    for lists in ([(64, a, b, 0), (64, c, b, 0)], [(64, a, a, 0), (64, a, a, 0)], [(64, a, b, 0), (64, b, c, 0)], [(64, a, a + 4, 0)],
                  [(64, a, b, 0), (2, c, b + 252, lp.LP_F16)], [(64, a, (1 << 20) - 252, 0)], [(64, 1 << 20, 1 << 20, 0)]):
        assert clip(lists) == lp.LP_ERR_INVALID_ARG and b"overlap" in lib.lp_last_error(), lists
    assert clip([(1 << 49, a, b, 0)]) == lp.LP_ERR_UNSUPPORTED
    n = C.c_size_t(7)
    arr = (lp._Gradient * 1)(lp._Gradient(*good))
    assert lib.lp_grad_norm_workspace_bytes(1, arr, C.byref(n)) == lp.LP_OK and n.value == 0
    assert lib.lp_grad_norm_workspace_bytes(1, arr, None) == lp.LP_ERR_INVALID_ARG
    assert lib.lp_grad_norm(1, arr, None, None, 0, None) == lp.LP_ERR_INVALID_ARG
