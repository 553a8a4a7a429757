"""A block's norms, join and dropout over more rows than the workgroups of a launch take at once, so that each takes several
in turn and some have one turn less, against the formulas in 64 bits: below and above 512 channels, where a row takes a
workgroup of its own."""
import numpy as np
import pytest
import torch

import gpu_common as H
import paper_2407_01781_amd as fx
import rows_reference as R
import test_gpu_block as T

pytestmark = pytest.mark.gpu
U = R.U


def _mask(rows, c, p, seed, offset):
    """R.keep_mask for many rows: the same whole numbers, all rows at once."""
    low, u = 0xFFFFFFFF, np.uint64
    full = lambda v: np.full((rows, (c + 7) // 8), v, u)
    w = [np.arange((c + 7) // 8, dtype=u)[None, :] + full(0), np.arange(rows, dtype=u)[:, None] + full(0), full(offset & low), full(offset >> 32 & low)]
    k = [seed & low, seed >> 32 & low]
    for _ in range(7):
        a, b = w[0] * u(0xD2511F53), w[2] * u(0xCD9E8D57)
        w = [(b >> u(32)) ^ w[1] ^ u(k[0]), b & u(low), (a >> u(32)) ^ w[3] ^ u(k[1]), a & u(low)]
        k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
    halves = np.stack([h for v in w for h in (v & u(0xFFFF), v >> u(16))], 2).reshape(rows, -1)[:, :c]
    return halves >= int(p * 65536 + 0.5)


@pytest.fixture
def many_rows(monkeypatch):
    a = R.keep_mask(19, 29, 0.3, 2 ** 63 + 7, 2 ** 40 + 1)
    assert np.array_equal(a, _mask(19, 29, 0.3, 2 ** 63 + 7, 2 ** 40 + 1))
    monkeypatch.setattr(R, "keep_mask", _mask)


# rows of the workgroups of one launch on 256 compute units -- forward 8,192 workgroups of 256 threads below 512 channels
# (33,001 x 512: 8,251 are needed), 16,384 of a row at 520 channels, 4,096 at 4,096; gradients of the join 512 below, 1,024 at
# 520, 256 at 4,096
@pytest.mark.parametrize("rows,c,dtype", [(40_003, 24, "f32"), (33_001, 512, "bf16"), (17_001, 520, "f16"), (2_500, 520, "f32"), (700, 4_096, "bf16"),
                                          (4_501, 2_100, "bf16")])
def test_join(rows, c, dtype, many_rows):
    T._join_case(rows, c, dtype, "f32", False, True, "silu", True, True, True, 0.1)


@pytest.mark.parametrize("rows,c,dtype", [(66_001, 256, "bf16"), (17_001, 520, "f32"), (5_003, 4_096, "f16"), (1_100, 4_095, "bf16")])
def test_norm(rows, c, dtype):
    x, rx = T._draw(91, rows, c, dtype, std=2.0)
    g, rg = T._draw(92, rows, c, dtype)
    w, rw = T._vec(93, c, "f32")
    out = H.nan_filled((rows, c), x.dtype)
    ref = R.norm(rx, rw, 1e-5)
    R.check(T._f64(fx.rms_norm_fwd(x, w, 1e-5, out=out)), ref, T._k(c) * np.abs(ref), dtype, "norm")
    gx, gw = fx.rms_norm_bwd(g, x, w, 1e-5)
    want, terms = R.norm_grad(rg, rx, rw, 1e-5)
    Ex, Ew = T._norm_grad_bound(np.zeros_like(rg), rg, rx, rw, 1e-5)
    R.check(T._f64(gx), want, Ex, dtype, "gx")
    T._sum_check(T._f64(gw), terms, Ew, "f32", "gweight")
    y = x.clone()
    assert torch.equal(fx.rms_norm_fwd(y, w, 1e-5, out=y), out)


@pytest.mark.parametrize("rows,c,dtype", [(300_007, 64, "bf16"), (70_001, 200, "f16"), (17_003, 520, "f32"), (4_301, 4_095, "bf16")])
def test_dropout(rows, c, dtype):
    x, rx = T._draw(94, rows, c, dtype)
    res, rres = T._draw(95, rows, c, dtype)
    ref = np.where(_mask(rows, c, 0.25, 77, 78), rx * R.drop_factor(0.25), 0.0)
    R.check(T._f64(fx.dropout(x, 0.25, 77, 78)), ref, U * np.abs(ref), dtype)
    R.check(T._f64(fx.dropout(x, 0.25, 77, 78, residual=res)), ref + rres, 2 * U * (np.abs(ref) + np.abs(rres)), dtype)
    y = x.clone()
    assert torch.equal(fx.dropout(y, 0.25, 77, 78, residual=res, out=y), fx.dropout(x, 0.25, 77, 78, residual=res))
