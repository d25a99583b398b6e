"""Strides whose product with a side leaves 64 bits are refused before anything touches a GPU: a reach that wraps
around would hide that what is written overlaps what is read."""
import ctypes as C

import pytest

from paper_2608_21607_gb300 import build as B
from paper_2608_21607_gb300 import nmd as N

P = 1 << 20   # an address that nothing reads: the calls end before
FAR = 1 << 40


@pytest.fixture(scope="module")
def L():
    B.build()
    return N.lib()


def ortho(L, rows, cols, rs, cs, out, ors, ocs):
    k = (C.c_double * 3)(3.4, -4.8, 2.0)
    return L.nmd_orthogonalize(P, 0, rows, cols, rs, cs, 5, k, 1e-7, out, ors, ocs, None, 0, None)


def muon(L, rows, cols, w, g, m):
    k = (C.c_double * 3)(3.4, -4.8, 2.0)
    keep = [N.nmd_matrix(*v) for v in (w, g, m)]
    return L.nmd_muon_step(*map(C.addressof, keep), rows, cols, 0.1, 0.9, 1, 0.0, 1.0, 5, k, 1e-7, None, 0, None)


# sides times strides of 2^63 (negative), 2^64 (back to nothing) and just below
@pytest.mark.parametrize("rows,rs", [((1 << 23) + 1, FAR), ((1 << 24) + 1, FAR), ((1 << 31) - 1, FAR), ((1 << 22) + 1, FAR)])
@pytest.mark.parametrize("turned", [False, True])
def test_reach_past_64_bits(L, rows, rs, turned):
    def two(a, b):
        return (b, a) if turned else (a, b)

    n, st = two(rows, 4), two(rs, 1)
    # what is written lies in the second row (or column) of what is read
    assert ortho(L, *n, *st, P + 4 * rs, *two(4, 1)) == N.NMD_ERR_INVALID
    assert ortho(L, *n, *two(4, 1), P + 16, *st) == N.NMD_ERR_INVALID
    far, near = (P, 0, *st), (P + 4 * rs, 0, *two(4, 1))
    apart = (1 << 62, 0, *two(4, 1))
    for matrices in ((far, near, apart), (near, far, apart), (apart, near, far), (far, apart, near)):
        assert muon(L, *n, *matrices) == N.NMD_ERR_INVALID


def test_reach_of_both_strides(L):
    # each by itself fits
    assert ortho(L, 1 << 14, 1 << 14, FAR, 1 << 39, P + 4 * FAR, 1 << 14, 1) == N.NMD_ERR_INVALID


def test_far_strides_that_fit(L):
    """Far apart, but nothing overlaps: only the workspace is missing."""
    assert ortho(L, 2, 4, FAR, 1, P + 64, 4, 1) == N.NMD_ERR_INVALID        # between the two rows
    assert ortho(L, 2, 4, FAR, 1, P + 4 * FAR + 64, 4, 1) == N.NMD_ERR_WORKSPACE
    assert ortho(L, 1 << 20, 4, 4, 1, P + (1 << 24), 4, 1) == N.NMD_ERR_WORKSPACE
    assert ortho(L, 1, 4, FAR, 1, P + 64, 4, 1) == N.NMD_ERR_WORKSPACE
