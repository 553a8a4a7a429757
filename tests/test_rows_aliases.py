"""CPU-only: single steps of the recurrence and a block's join refuse outputs that lie on each other or where the kernel
still reads, on the host, before anything reaches a GPU."""
import ctypes as C

import pytest

from paper_2407_01781_amd import binding as B

AT = [C.c_void_p((i + 1) << 20) for i in range(8)]          # never followed: every call here is refused


def _refused(status, name, *args):
    assert getattr(B.lib, name)(*args) == status
    assert name.encode() in B.lib.fx_last_error()


def _step(h=AT[2], s=AT[3], n=AT[4], rows=5, c=12):
    return "fx_gated_scan_step", AT[0], c, AT[1], c, 0, rows, c, s, n, h, c, None


@pytest.mark.parametrize("c", [5, 12, 16])
def test_step(c):
    _refused(-1, *_step(h=AT[0], c=c))
    _refused(-1, *_step(h=AT[1], c=c))
    # the new states may be the old ones in place, not half of them
    for off in (4, 4 * 5 * c - 4):
        _refused(-1, *_step(n=C.c_void_p(AT[3].value + off), c=c))
        _refused(-1, *_step(n=C.c_void_p(AT[3].value - off), c=c))
