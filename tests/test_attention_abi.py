"""CPU-only: attention, its gradients, the cache and the step refuse bad arguments on the host, with a status and a text, before
anything reaches a GPU."""
import ctypes as C
import math

import pytest

from paper_2407_01781_amd import binding as B

P = [C.c_void_p((i + 1) << 20) for i in range(12)]          # never followed: every call here is refused
ODD = C.c_void_p((1 << 20) + 1)
SEQS = (C.c_int64 * 64)()           # the members that a refusal reads: rows, longest, B


def _seqs(rows=100, batch=1):
    s = (C.c_int64 * 64)()
    s[0], s[1] = rows, rows
    C.cast(s, C.POINTER(C.c_int32))[4] = batch
    return s


def _refused(status, name, *args):
    assert getattr(B.lib, name)(*args) == status, B.lib.fx_last_error()
    assert name.encode() in B.lib.fx_last_error()


def _attention(**kw):
    a = dict(q_seqs=C.addressof(S), kv_seqs=None, dt=2, heads=4, kv_heads=2, dim=64, causal=0, scale=0.125, d_q=P[0].value, d_k=P[1].value, d_v=P[2].value, ld_q=256, hs_q=64,
             ld_k=128, hs_k=64, ld_v=128, hs_v=64)
    return B._Attention(**{**a, **kw})


S, OTHER = _seqs(), _seqs(50, 3)


def _fwd(a, out=P[3], ld=256, hs=64, lse=P[4]):
    return "fx_attention_fwd", None if a is None else C.byref(a), out, ld, hs, lse, None


BAD = [dict(q_seqs=None), dict(dt=3), dict(dt=-1), dict(heads=0), dict(kv_heads=0), dict(heads=3), dict(heads=-4), dict(dim=0), dict(scale=math.nan), dict(scale=math.inf),
       dict(kv_seqs=C.addressof(OTHER)), dict(d_q=None), dict(d_k=None), dict(d_v=None), dict(d_q=ODD.value), dict(ld_q=63), dict(hs_q=63), dict(ld_k=0), dict(hs_v=-64), dict(ld_v=-128)]


@pytest.mark.parametrize("kw", BAD, ids=lambda kw: next(iter(kw)))
def test_description(kw):
    _refused(-1, *_fwd(_attention(**kw)))
    _refused(-1, *_bwd(_attention(**kw)))


def _bwd(a, out=P[3], lse=P[4], go=P[5], gl=None, gq=P[6], gk=P[7], gv=P[8], ld=256, kld=128):
    return "fx_attention_bwd", None if a is None else C.byref(a), out, ld, 64, lse, go, ld, 64, gl, gq, ld, 64, gk, kld, 64, gv, kld, 64, None


def test_forward():
    _refused(-1, *_fwd(None))
    for bad in (_fwd(_attention(), out=None), _fwd(_attention(), out=ODD), _fwd(_attention(), ld=60), _fwd(_attention(), hs=60), _fwd(_attention(), lse=ODD),
                _fwd(_attention(), out=P[0]), _fwd(_attention(), out=P[1]), _fwd(_attention(), out=P[2]),
                _fwd(_attention(), ld=192, hs=64),              # rows of four heads closer than they are wide
                _fwd(_attention(), ld=64, hs=64 * 99)):         # heads of a hundred rows closer than those
        _refused(-1, *bad)
    _refused(-5, *_fwd(_attention(dim=257, ld_q=2056, hs_q=257, ld_k=514, hs_k=257, ld_v=514, hs_v=257), ld=2056, hs=257))
    _refused(-5, *_fwd(_attention(ld_q=1 << 47)))
    _refused(-5, *_fwd(_attention(heads=1 << 17, kv_heads=1)))


def test_backward():
    _refused(-1, *_bwd(None))
    for bad in (_bwd(_attention(), out=None), _bwd(_attention(), lse=None), _bwd(_attention(), go=None), _bwd(_attention(), lse=ODD), _bwd(_attention(), gl=ODD),
                _bwd(_attention(), gq=ODD), _bwd(_attention(), gk=P[1]), _bwd(_attention(), gv=P[7]), _bwd(_attention(), gq=P[5]), _bwd(_attention(), gq=P[3]),
                _bwd(_attention(), ld=200), _bwd(_attention(), kld=100)):
        _refused(-1, *bad)


def _cache(**kw):
    a = dict(d_k=P[0].value, d_v=P[1].value, d_k_exp=None, d_v_exp=None, d_table=P[2].value, ld_table=8, table_cols=8, pages=10, page_rows=16, store=2, kv_heads=2, dim=64)
    return B._Cache(**{**a, **kw})


def _write(c, q=None, rows=5, start=P[3], dt=2, k=P[4], v=P[5], ld=128, hs=64):
    return "fx_cache_write", None if c is None else C.byref(c), q, rows, start, dt, k, ld, hs, v, ld, hs, None


def _read(c, q=C.addressof(S), start=P[3], dt=2, k=P[4], v=P[5], ld=128, hs=64):
    return "fx_cache_read", None if c is None else C.byref(c), q, start, dt, k, ld, hs, v, ld, hs, None


def _step(c, rows=5, lens=P[3], most=0, dt=2, heads=4, scale=0.125, q=P[4], out=P[5], lse=P[6], ld=256, hs=64):
    return "fx_attention_step", None if c is None else C.byref(c), rows, lens, most, dt, heads, scale, q, ld, hs, out, ld, hs, lse, None


E4 = dict(store=3, d_k_exp=P[6].value, d_v_exp=P[7].value)


@pytest.mark.parametrize("call", [_write, _read, _step], ids=["write", "read", "step"])
def test_cache(call):
    _refused(-1, *call(None))
    for kw in (dict(d_k=None), dict(d_v=None), dict(d_k=P[0].value + 8), dict(d_v=P[0].value), dict(d_table=None), dict(d_table=ODD.value), dict(ld_table=7), dict(table_cols=-1),
               dict(pages=-1), dict(page_rows=0), dict(store=4), dict(store=-1), dict(kv_heads=0), dict(dim=0), dict(store=3), dict(d_k_exp=P[6].value),
               dict(store=3, d_k_exp=P[6].value, d_v_exp=P[6].value)):
        _refused(-1, *call(_cache(**kw)))
    _refused(-2, *call(_cache(store=1)))                # rows of bf16 into pages of f16
    _refused(-1, *call(_cache(), dt=3))
    _refused(-5, *call(_cache(dim=257), ld=1 << 12, hs=1 << 10))
    _refused(-5, *call(_cache(pages=1 << 27)))          # 2^32 rows of pages and heads
    for kw in (dict(ld=63), dict(hs=63)):
        _refused(-1, *call(_cache(**E4), **kw))


def test_rows_of_the_cache():
    for bad in (_write(_cache(), rows=-1), _write(_cache(), q=C.addressof(S), rows=99), _write(_cache(), start=None), _write(_cache(), start=ODD), _write(_cache(), k=None),
                _write(_cache(), v=ODD), _read(_cache(), q=None), _read(_cache(), start=None), _read(_cache(), k=None), _read(_cache(), v=P[4]), _read(_cache(), ld=100),
                _step(_cache(), rows=-1), _step(_cache(), most=-1), _step(_cache(), heads=3), _step(_cache(), heads=0), _step(_cache(), scale=math.nan), _step(_cache(), lens=None),
                _step(_cache(), lens=ODD), _step(_cache(), lse=ODD), _step(_cache(), q=None), _step(_cache(), out=None), _step(_cache(), out=P[4]), _step(_cache(), ld=200)):
        _refused(-1, *bad)
    _refused(-5, *_write(_cache(), rows=1 << 31))
    _refused(-5, *_step(_cache(), rows=1 << 40))
    _refused(-5, *_step(_cache(), rows=(1 << 63) - 1))
    _refused(-5, *_step(_cache(table_cols=1 << 28, ld_table=1 << 28)))


def test_threads_of_a_step_are_counted_in_32_bits():
    """2^24 workgroups of 256 threads would wrap to none; 34 heads that share a key head are three workgroups."""
    for rows, heads in ((1 << 24, 4), (1 << 23, 4), (1 << 22, 68)):
        _refused(-5, *_step(_cache(), rows=rows, heads=heads, ld=heads * 64))


@pytest.mark.parametrize("struct,offsets", [(B._Attention, {"dt": 16, "heads": 20, "causal": 32, "scale": 36, "d_q": 40, "ld_q": 64, "hs_v": 104}),
                                            (B._Cache, {"d_k_exp": 16, "d_table": 32, "ld_table": 40, "table_cols": 48, "store": 60, "dim": 68})])
def test_descriptions_lie_as_the_header_says(struct, offsets):
    """Offsets of the members, counted from the header."""
    assert {k: getattr(struct, k).offset for k in offsets} == offsets
