"""Sizes beyond what the products can count: refused, by name, before anything touches a device."""
import ctypes as C

import pytest

from paper_2605_01989_b200 import binding as dblp

ECAPACITY = -3
MOST = (1 << 31) - 1
A = 1 << 40                                            # addresses that are never read, far enough apart


def matrix(data, cols, off=0):
    return C.byref(dblp.dblp_matrix_t(data + 2 * off, (cols + 15) // 16 * 16 + off, 1))


def text():
    return dblp.lib().dblp_last_error().decode()


@pytest.mark.parametrize("n,i,o,fits", [(MOST, MOST, MOST, False), (MOST, 64, MOST, False), (MOST, 64, 64, True), (1 << 20, 1 << 21, 64, True)])
def test_workspaces_are_whole_numbers_or_refused(n, i, o, fits):
    """Rows off 16 bytes: the copies of x and w alone, and for the largest sizes about 2^64 bytes."""
    l = dblp.dblp_linear_t(n, i, o, 1, 1, 0, 0, 0)
    f, g = C.c_size_t(), C.c_size_t()
    rc = dblp.lib().dblp_linear_workspace_bytes(C.byref(l), matrix(A, i, 1), matrix(A, o, 1), matrix(A, o, 1), C.byref(f), C.byref(g))
    if fits:
        assert rc == 0 and f.value >= 2 * (n * i + i * o) and g.value >= 2 * (n * o + i * o) and max(f.value, g.value) < 1 << 62
    else:
        assert rc == ECAPACITY and "2^62" in text()


@pytest.mark.parametrize("n,o", [(MOST, MOST), (1 << 30, 1 << 23)])
def test_more_tiles_than_can_be_counted(n, o):
    l = dblp.dblp_linear_t(n, 64, o, 1, 1, 0, 0, 0)
    rc = dblp.lib().dblp_linear(C.byref(l), matrix(A, 64), matrix(A + (1 << 50), o), None, None, None, matrix(A + (1 << 55), o), A, 1 << 62, None)
    assert rc == ECAPACITY and "2^30 tiles" in text(), (rc, text())
