"""CPU-only: the operators around the convolution refuse bad arguments on the host, with a status and a text, before
anything reaches a GPU."""
import ctypes as C
import math

import pytest

from paper_2407_01781_amd import binding as B

P = C.c_void_p(256)          # never followed: every call here is refused
ODD = C.c_void_p(257)


def _refused(status, name, *args):
    assert getattr(B.lib, name)(*args) == status
    assert name.encode() in B.lib.fx_last_error()


def _offsets(*pairs):
    return (C.c_int64 * (2 * len(pairs)))(*[v for p in pairs for v in p])


def test_sequences():
    h = C.c_void_p()
    out = C.byref(h)
    _refused(-1, "fx_build_sequences", None, 1, 4, None, out)
    _refused(-1, "fx_build_sequences", _offsets((0, 4)), 1, 4, None, None)
    _refused(-1, "fx_build_sequences", _offsets((0, 4)), -1, 4, None, out)
    _refused(-1, "fx_build_sequences", None, 0, 4, None, out)                       # rows of no sequence
    _refused(-1, "fx_build_sequences", _offsets((0, 4)), 1, 5, None, out)           # rows behind the last
    _refused(-1, "fx_build_sequences", _offsets((1, 4)), 1, 4, None, out)           # rows before the first
    _refused(-1, "fx_build_sequences", _offsets((0, 2), (3, 4)), 2, 4, None, out)
    _refused(-1, "fx_build_sequences", _offsets((0, 2), (2, 1)), 2, 1, None, out)
    _refused(-5, "fx_build_sequences", _offsets((0, 1 << 31)), 1, 1 << 31, None, out)
    assert not h.value
    B.lib.fx_sequences_destroy(None)


def test_scan():
    _refused(-1, "fx_gated_scan_fwd", None, P, 8, P, 8, 0, 8, 0, None, P, 8, None, None)
    _refused(-1, "fx_gated_scan_bwd", None, P, 8, P, 8, P, 8, P, 8, 0, 8, 0, None, None, P, 8, P, 8, None, None)
    step = lambda x=P, ld=8, dt=0, rows=2, c=8, s=P, n=P, h=P: ("fx_gated_scan_step", x, ld, P, 8, dt, rows, c, s, n, h, 8, None)
    _refused(-5, *step(ld=1 << 25, c=(1 << 24) + 1))
    for bad in (step(x=None), step(x=ODD), step(ld=7), step(dt=3), step(rows=-1), step(c=0), step(s=None), step(n=None), step(h=None)):
        _refused(-1, *bad)


def test_norm():
    fwd = lambda x=P, ld=8, dt=0, rows=2, c=8, w=P, vdt=0, eps=1e-6, o=P, lo=8: ("fx_rms_norm_fwd", x, ld, dt, rows, c, w, vdt, eps, o, lo, None)
    for bad in (fwd(x=None), fwd(x=ODD), fwd(ld=7), fwd(dt=-1), fwd(rows=-1), fwd(c=0), fwd(w=ODD), fwd(vdt=2), fwd(eps=-1.0), fwd(eps=math.nan),
                fwd(eps=math.inf), fwd(o=None), fwd(lo=7)):
        _refused(-1, *bad)
    _refused(-5, *fwd(c=4097, ld=4097, lo=4097))
    _refused(-5, *fwd(rows=1 << 31))
    bwd = lambda g=P, x=P, gx=P, ld=8, gw=P: ("fx_rms_norm_bwd", g, ld, x, ld, 0, 2, 8, P, 0, 1e-6, gx, ld, gw, None)
    for bad in (bwd(g=None), bwd(x=None), bwd(gx=ODD), bwd(gw=ODD), bwd(ld=7)):
        _refused(-1, *bad)


def _join(**kw):
    a = dict(rows=2, C=8, dt=0, vec_dt=0, act=1, d_y=256, d_gate=256, ld_y=8, ld_gate=8, d_post=256, d_scale=256, d_next=256, eps=1e-6)
    return B._BlockJoin(**{**a, **kw})


def test_join():
    fwd = lambda b, x=P, o=P, n=P, ld=8: ("fx_block_join_fwd", b and C.byref(b), x, ld, o, ld, n, ld, None)
    _refused(-1, *fwd(None))
    for kw in (dict(rows=-1), dict(C=0), dict(dt=5), dict(vec_dt=1), dict(act=2), dict(d_y=None), dict(d_y=257), dict(ld_y=7), dict(d_gate=257),
               dict(ld_gate=3), dict(d_post=258), dict(d_scale=258), dict(d_next=258), dict(eps=-1.0), dict(p=-0.5), dict(p=1.5), dict(p=math.nan),
               dict(d_offset=260)):
        _refused(-1, *fwd(_join(**kw)))
    for bad in (fwd(_join(), x=None), fwd(_join(), o=None), fwd(_join(), n=None), fwd(_join(), ld=7), fwd(_join(d_next=None))):
        _refused(-1, *bad)
    _refused(-5, *fwd(_join(C=5000, ld_y=5000, ld_gate=5000), ld=5000))
    bwd = lambda b, go=P, gn=P, o=P, gg=P, gp=P, gs=P, gnx=P: ("fx_block_join_bwd", C.byref(b), go, 8, gn, 8, o, 8, P, 8, P, 8, gg, 8, gp, gs, gnx, None)
    for bad in (bwd(_join(), go=None, gn=None), bwd(_join(), o=None), bwd(_join(d_next=None)), bwd(_join(d_next=None), gn=None),
                bwd(_join(d_gate=None)), bwd(_join(d_post=None)), bwd(_join(d_scale=None)), bwd(_join(), go=ODD), bwd(_join(), gp=ODD)):
        _refused(-1, *bad)


def test_dropout():
    call = lambda x=P, ld=8, dt=0, rows=2, c=8, p=0.5, d=None, r=None, o=P: ("fx_dropout", x, ld, dt, rows, c, p, 1, 2, d, r, 8, o, 8, None)
    for bad in (call(x=None), call(ld=7), call(dt=9), call(rows=-2), call(c=0), call(p=-1e-9), call(p=1.0001), call(p=math.nan), call(d=C.c_void_p(260)),
                call(r=ODD), call(o=None)):
        _refused(-1, *bad)


@pytest.mark.parametrize("name", ["dt", "vec_dt", "act", "d_offset", "eps"])
def test_description_lies_as_the_header_says(name):
    """Offsets of fx_block_join's members, counted from the header: 8 + 4 x 4, 2 pointers, 2 strides, 4 pointers, 2 + 1 words."""
    assert getattr(B._BlockJoin, name).offset == {"dt": 12, "vec_dt": 16, "act": 20, "d_offset": 80, "eps": 112}[name]
