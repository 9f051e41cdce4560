"""Host-side checks of how many rows and outputs one projection on 8-bit integers takes (the pointers are never dereferenced)."""
import ctypes

import pytest

from paper_2607_27591_amd import prox

FAKE, UNSUPPORTED = 0x100000, 2


@pytest.mark.parametrize("rows,n", [(1 << 22, 130817), (524033, 1 << 20), (1 << 22, 1 << 20)])
def test_linear_w8_refuses_more_tiles_than_a_grid_holds(rows, n):
    q = prox._W8Linear(prox.BF16, n, 16, FAKE, 1 << 45)
    assert prox.lib().prox_linear_w8(ctypes.byref(q), FAKE, 16, FAKE, rows, None, FAKE, n, None) == UNSUPPORTED
