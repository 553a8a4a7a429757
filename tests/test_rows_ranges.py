"""CPU-only: numbers of rows beyond what a launch holds are refused before they meet in a product that wraps."""
import ctypes as C

import pytest

from paper_2407_01781_amd import binding as B

P, Q, R = (C.c_void_p((i + 1) << 20) for i in range(3))          # never followed


@pytest.mark.parametrize("rows,c", [((1 << 39) // 8, 64), (1 << 60, 128), (1 << 61, 64), ((1 << 63) - 1, 1)])
def test_step(rows, c):
    assert B.lib.fx_gated_scan_step(P, c, P, c, 0, rows, c, Q, Q, R, c, None) == -5
    assert b"fx_gated_scan_step" in B.lib.fx_last_error()
