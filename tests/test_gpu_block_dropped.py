"""A block's join where values that are not finite are dropped: a dropped value leaves 0, so outputs and gradients are those
of the same call with any finite number in its place, at widths whose pieces fill a power of two of lanes and at widths
that leave lanes of a row idle, with rows that do not fill a wave's or a workgroup's last turn."""
import numpy as np
import pytest
import torch

import gpu_common as H
import paper_2407_01781_amd as fx
import rows_reference as R
import test_gpu_block as T

pytestmark = pytest.mark.gpu
U = R.U
SEED, OFFSET, P, EPS = 0xC0FFEE, (3 << 32) + 5, 0.4, 1e-5
BAD = [float("inf"), float("-inf"), float("nan")]


def _inputs(c, dtype, spoil):
    """Every second row and the last have values that are not finite wherever dropout drops, in the tensors of `spoil`; the
    reference's copies have zeros there."""
    n = 7 if c > 512 else 33
    keep = R.keep_mask(n, c, P, SEED, OFFSET)
    rows = np.zeros((n, 1), bool)
    rows[::2] = rows[-1] = True
    at = ~keep & rows
    assert at.any() and at[-1].any() and at[:, -8:].any()
    d = {}
    for s, (name, std) in enumerate((("x", 1.5), ("y", 3.0), ("gate", 1.5), ("gout", 1.0), ("gnorm", 1.0))):
        t, v = T._draw(70 + s, n, c, dtype, False, std)
        if name in spoil:
            v = np.where(at, 0.0, v)
            bad = torch.tensor(np.resize(BAD, at.sum()), dtype=t.dtype, device="cuda")
            t[torch.from_numpy(at).cuda()] = bad
        d[name] = (t, v)
    return n, keep * R.drop_factor(P), at, d


WIDTHS = [5, 24, 40, 45, 48, 64, 96, 100, 512, 520, 1000]


@pytest.mark.parametrize("c", WIDTHS)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act", ["silu", "sigmoid"])
def test_outputs(c, dtype, act):
    n, keep, _, d = _inputs(c, dtype, ("gate",))
    (wp, rp), (ws, rs), (wn, rn) = (T._vec(s, c, "f32") for s in (81, 82, 83))
    x, rx = d["x"]
    for post, rpost in ((None, None), (wp, rp)):
        out, norm = fx.block_join_fwd(x, d["y"][0], gate=d["gate"][0], act=act, post_weight=post, scale=ws, next_weight=wn, eps=EPS, p=P,
                                      seed=SEED, offset=OFFSET)
        ref, rnorm = R.join(rx, d["y"][1], d["gate"][1], act, rpost, rs, rn, EPS, keep)
        Eo = (T._k(c) + (2 * np.abs(d["gate"][1]) + 16) * U) * np.abs(ref - rx) + U * np.abs(ref)
        R.check(T._f64(out), ref, Eo, dtype, "out")
        r = 1 / np.sqrt((ref * ref).mean(1, keepdims=True) + EPS)
        En = np.abs(rn) * r * (Eo + np.abs(ref) * (T._k(c) + r * np.sqrt((Eo * Eo).mean(1, keepdims=True))))
        R.check(T._f64(norm), rnorm, En, dtype, "norm")
