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


def test_join():
    b = B._BlockJoin(rows=3, C=8, dt=0, vec_dt=0, act=1, d_y=AT[0].value, d_gate=AT[1].value, ld_y=8, ld_gate=8, d_next=AT[7].value, eps=1e-6)
    _refused(-1, "fx_block_join_fwd", C.byref(b), AT[2], 8, AT[3], 8, AT[3], 8, None)
    bwd = lambda gx, gy, gg: ("fx_block_join_bwd", C.byref(b), AT[2], 8, AT[3], 8, AT[4], 8, gx, 8, gy, 8, gg, 8, None, None, None, None)
    for which in ((AT[5], AT[5], None), (AT[5], AT[6], AT[5]), (None, AT[6], AT[6])):
        _refused(-1, *bwd(*which))
