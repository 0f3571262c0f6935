"""Argument errors of the norm and of the orthogonalised updates are statuses before anything touches a GPU.  CPU only."""
import ctypes as C

import pytest
import torch


@pytest.fixture()
def lib():
    import paper_2404_19760_amd as lp
    return lp, lp._lib


def _norm(lp, **kw):
    q = lp._GroupNorm(1, 10, 8, 2, lp.LP_ACT_SILU, 1e-5, lp.LP_F32, lp.LP_F32, 0, 0, None, None, None)
    for k, v in kw.items():
        setattr(q, k, v)
    return q


def test_group_norm_refusals(lib):
    lp, lib = lib
    one = C.c_void_p(4096)

    def fwd(q):
        return lib.lp_group_norm_fwd(q and C.byref(q), one, one, None, None, 0, None)

    def bwd(q):
        return lib.lp_group_norm_bwd(q and C.byref(q), one, one, one, one, None, None, None, 0, None)

    for call in (fwd, bwd):
        assert call(None) == lp.LP_ERR_INVALID_ARG and b"NULL" in lib.lp_last_error()
        for kw, word in ((dict(N=-1), b"N"), (dict(P=-1), b"P"), (dict(C=0), b"divide"), (dict(G=0), b"divide"), (dict(G=3), b"divide"),
                         (dict(act=4), b"act"), (dict(act=-1), b"act"), (dict(eps=-1.0), b"eps"), (dict(eps=float("inf")), b"eps"),
                         (dict(x_dtype=3), b"dtype"), (dict(y_dtype=-1), b"dtype"), (dict(x_stride=7), b"stride"), (dict(y_stride=-8), b"stride")):
            assert call(_norm(lp, **kw)) == lp.LP_ERR_INVALID_ARG and word in lib.lp_last_error(), kw
        assert call(_norm(lp, x_dtype=lp.LP_BF16)) == lp.LP_ERR_UNSUPPORTED
        assert call(_norm(lp, N=1 << 40, P=1 << 40)) == lp.LP_ERR_UNSUPPORTED
        assert call(_norm(lp, N=0)) == lp.LP_OK and call(_norm(lp, P=0)) == lp.LP_OK   # nothing to do
    assert lib.lp_group_norm_fwd(C.byref(_norm(lp)), None, one, None, None, 0, None) == lp.LP_ERR_INVALID_ARG
    assert lib.lp_group_norm_bwd(C.byref(_norm(lp)), one, None, one, one, None, None, None, 0, None) == lp.LP_ERR_INVALID_ARG


def test_orthogonalise_refusals(lib):
    lp, lib = lib
    orth = lp._Orth(5, None, 1e-7)
    good = lp._Matrices(1, 8, 8, 4096, 4096, lp.LP_F32)

    def run(m, o=orth, n=1):
        return lib.lp_orthogonalize(n, m and C.byref(m), o and C.byref(o), None, 0, None)

    assert run(good, None) == lp.LP_ERR_INVALID_ARG and run(None) == lp.LP_ERR_INVALID_ARG and run(good, n=-1) == lp.LP_ERR_INVALID_ARG
    for m, status in ((lp._Matrices(-1, 8, 8, 4096, 4096, 0), lp.LP_ERR_INVALID_ARG), (lp._Matrices(1, -8, 8, 4096, 4096, 0), lp.LP_ERR_INVALID_ARG),
                      (lp._Matrices(1, 8, 8, None, 4096, 0), lp.LP_ERR_INVALID_ARG), (lp._Matrices(1, 8, 8, 4096, None, 0), lp.LP_ERR_INVALID_ARG),
                      (lp._Matrices(1, 8, 8, 4096, 4096, 5), lp.LP_ERR_INVALID_ARG), (lp._Matrices(1, 70000, 8, 4096, 4096, 0), lp.LP_ERR_UNSUPPORTED),
                      (lp._Matrices(1 << 21, 8, 8, 4096, 4096, 0), lp.LP_ERR_UNSUPPORTED)):
        assert run(m) == status and b"lists[0]" in lib.lp_last_error()
    for o in (lp._Orth(0, None, 0.0), lp._Orth(17, None, 0.0), lp._Orth(5, None, -1.0), lp._Orth(5, None, float("nan"))):
        assert run(good, o) == lp.LP_ERR_INVALID_ARG
    assert run(lp._Matrices(0, 8, 8, None, None, 0)) == lp.LP_OK and run(None, n=0) == lp.LP_OK   # nothing to do
    large = lp._Matrices(1, 300, 300, 4096, 4096, lp.LP_F32)
    assert run(large) == lp.LP_ERR_WORKSPACE
    n = C.c_size_t(7)
    assert lib.lp_orthogonalize_workspace_bytes(1, C.byref(good), C.byref(n)) == lp.LP_OK and n.value == 0
    assert lib.lp_orthogonalize_workspace_bytes(1, C.byref(large), C.byref(n)) == lp.LP_OK and n.value > 300 * 300 * 8
    assert lib.lp_orthogonalize_workspace_bytes(1, C.byref(large), None) == lp.LP_ERR_INVALID_ARG


def test_muon_refusals(lib):
    lp, lib = lib
    w = lp._MuonWeights(1, 300, 300, 4096, 4096, 4096)

    def run(q, w=w):
        return lib.lp_muon_step(1, w and C.byref(w), q and C.byref(q), None, 0, None)

    def muon(**kw):
        q = lp._Muon(0.1, 0.9, 0.0, 1, lp.LP_MUON_SCALE_ASPECT, lp._Orth(5, None, 1e-7))
        for k, v in kw.items():
            setattr(q, k, v)
        return q

    assert run(None) == lp.LP_ERR_INVALID_ARG
    for kw in (dict(lr=float("nan")), dict(momentum=float("inf")), dict(weight_decay=float("nan")), dict(nesterov=2), dict(scale=3), dict(scale=-1)):
        assert run(muon(**kw)) == lp.LP_ERR_INVALID_ARG, kw
    assert run(muon(), lp._MuonWeights(1, 300, 300, 4096, None, 4096)) == lp.LP_ERR_INVALID_ARG
    assert run(muon()) == lp.LP_ERR_WORKSPACE


def test_binding_refuses_what_is_not_on_the_gpu(lib):
    lp, _ = lib
    x = torch.zeros(1, 10, 8)
    with pytest.raises(ValueError, match="GPU"):
        lp.group_norm_fwd(lp.GroupNorm(2), x)
    with pytest.raises(ValueError, match="GPU"):
        lp.orthogonalize([torch.zeros(4, 4)])
    with pytest.raises(ValueError, match="GPU"):
        lp.muon_step([torch.zeros(4, 4)], [torch.zeros(4, 4)], [torch.zeros(4, 4)], lr=0.1)
    with pytest.raises(ValueError, match="gradient"):
        lp.lp_muon_step([torch.zeros(4, 4)], [], [], None, lr=0.1)
    with pytest.raises(ValueError, match="every step"):
        lp._orth(3, [(1.0, 1.0, 1.0)], 0.0)
