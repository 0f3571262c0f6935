"""Blocks that a wave of the orthogonalisation turns over in its own LDS (paper_2404_19760_amd/csrc/lp_orth.hip), checked on the
CPU from the source: lanes store what other lanes read, no address of a single lane says so, and the compiler may exchange the two
unless a `wave_lds_fence` or a barrier stands between them.  Accesses are taken in the order in which they are written down, twice
over (the blocks come in a loop).  And the same of the workgroup's LDS: sums are exchanged between two barriers."""
import os
import re

import pytest

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2404_19760_amd", "csrc", "lp_orth.hip")


def _body(first, last):
    lines = [line.split("//")[0] for line in open(SRC).read().split("\n")]
    a = next(i for i, l in enumerate(lines) if re.search(first, l))
    return lines[a:next(i for i in range(a + 1, len(lines)) if re.search(last, lines[i]))]


def _events(lines):
    out = []
    for line in lines:
        if "wave_lds_fence()" in line or "__syncthreads()" in line:
            out.append("fence")
        elif re.search(r"\bturn\[.*\]\s*=[^=]", line):
            out.append("store")
        elif re.search(r"\bturn\[", line):
            out.append("read")
    return out


@pytest.mark.parametrize("first,last,accesses", [(r"void orth_product_kernel\(", r"^struct Plan", 4), (r"void small_steps\(", r"orth_small_kernel", 2)])
def test_a_fence_between_stores_and_reads_of_other_lanes(first, last, accesses):
    events = _events(_body(first, last))
    assert sum(e != "fence" for e in events) == accesses and {"store", "read"} <= set(events)
    open_access = None
    for e in events * 2:
        if e == "fence":
            open_access = None
        else:
            assert open_access in (None, e), "a store and a read of other lanes' values without a fence between them"
            open_access = e


def test_exchanged_sums_lie_between_barriers():
    """Everybody's loop is done before the sums go over its buffers, they are all there before they are read, and read before the
    waves' blocks go over them."""
    lines = _body(r"void orth_product_kernel\(", r"^struct Plan")
    where = lambda pattern: [i for i, l in enumerate(lines) if re.search(pattern, l)]  # noqa: E731
    barriers = where(r"__syncthreads\(\);")
    last_product, = where(r"if \(k == 0\) __syncthreads")
    give, = where(r"\*slot\(g, group, e\) = v")
    take, = where(r": \*slot\(group, g, e\)")
    first_turn = where(r"\bturn\[")[0]
    for a, b in ((last_product, give), (give, take), (take, first_turn)):
        assert any(a < i < b for i in barriers)
