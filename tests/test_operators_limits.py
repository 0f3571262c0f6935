"""Lists of the orthogonalised updates that are refused before anything touches a GPU.  CPU only."""
import ctypes as C

import pytest


@pytest.fixture()
def lp():
    import paper_2404_19760_amd as lp
    return lp


def _orthogonalize(lp, lists):
    arr = (lp._Matrices * len(lists))(*[lp._Matrices(*q) for q in lists])
    return lp._lib.lp_orthogonalize(len(lists), arr, C.byref(lp._Orth(5, None, 1e-7)), None, 0, None)


def _muon(lp, lists):
    arr = (lp._MuonWeights * len(lists))(*[lp._MuonWeights(*q) for q in lists])
    q = lp._Muon(0.1, 0.9, 0.0, 1, lp.LP_MUON_SCALE_ASPECT, lp._Orth(5, None, 1e-7))
    return lp._lib.lp_muon_step(len(lists), arr, C.byref(q), None, 0, None)


def test_lists_that_write_what_others_hold_are_refused(lp):
    """Matrices of different lists are worked on at the same time: nothing says whether a value is read before or after another
    list's result lies over it.  (8 x 8 matrices in fp32 take 256 bytes and no workspace.)"""
    a, b, c, d, e, f = (4096 * k for k in range(1, 7))
    for lists in ([(1, 8, 8, a, b, lp.LP_F32), (1, 8, 8, b, c, lp.LP_F32)],            # a result over another list's input
                  [(1, 8, 8, b, c, lp.LP_F32), (1, 8, 8, a, b, lp.LP_F32)],
                  [(1, 8, 8, a, c, lp.LP_F32), (1, 8, 8, b, c, lp.LP_F32)],            # two results
                  [(1, 8, 8, a, a, lp.LP_F32), (1, 8, 8, a, a, lp.LP_F32)],            # the same matrix twice
                  [(1, 8, 8, a, b, lp.LP_F32), (2, 8, 8, c, b - 256, lp.LP_F32)],      # the last value of a list, the first of another
                  [(1, 8, 8, a, a + 252, lp.LP_F32)],                                  # shifted over its own input
                  [(1, 8, 8, a + 126, a, lp.LP_BF16)],
                  [(1, 8, 8, a, a, lp.LP_F32), (1, 4, 4, b, c, lp.LP_F32), (1, 4, 4, d, a + 128, lp.LP_F16)]):
        assert _orthogonalize(lp, lists) == lp.LP_ERR_INVALID_ARG and b"overlap" in lp._lib.lp_last_error(), lists
    for lists in ([(1, 8, 8, a, b, c), (1, 8, 8, a, d, e)],                            # a weight twice
                  [(1, 8, 8, a, b, c), (1, 8, 8, d, e, c)],                            # a momentum twice
                  [(1, 8, 8, a, b, c), (1, 8, 8, d, a, f)],                            # a weight that is another list's gradient
                  [(1, 8, 8, a, a, c)], [(1, 8, 8, a, b, b)], [(1, 8, 8, a, b, a)],    # a list's own
                  [(1, 8, 8, a, b, a + 252)]):
        assert _muon(lp, lists) == lp.LP_ERR_INVALID_ARG and b"overlap" in lp._lib.lp_last_error(), lists


def _workspace_bytes(lp, *shapes):
    arr = (lp._Matrices * len(shapes))(*[lp._Matrices(*s, None, None, lp.LP_F32) for s in shapes])
    n = C.c_size_t(0)
    assert lp._lib.lp_orthogonalize_workspace_bytes(len(shapes), arr, C.byref(n)) == lp.LP_OK
    return n.value


@pytest.mark.parametrize("shape,divided", [((1, 300, 300), 0), ((8, 333, 1001), 0), ((2, 512, 512), 0), ((30, 2048, 512), 0),
                                           ((1, 100, 5001), 3 * 3), ((2, 300, 1400), 2 * 15 * 2)])
def test_workspace_has_room_for_parts_of_sums_only_where_sums_are_divided(lp, shape, divided):
    """X and X^T twice and A and B, as two fp16 parts and padded to 64, for every matrix; 4 KB of partial norms for each and some KB
    of descriptors; where the sums of X X^T are divided, 64 x 64 sums in fp32 a part."""
    count, rows, cols = shape
    m, n = ((min(rows, cols) + 63) // 64 * 64, (max(rows, cols) + 63) // 64 * 64)
    planes = count * (8 * m * n + 4 * m * m) * 2
    extra = _workspace_bytes(lp, shape) - planes - count * 4096
    if divided:
        assert divided * 64 * 64 * 4 <= extra <= 1 << 26
    else:
        assert 0 <= extra <= 8192
