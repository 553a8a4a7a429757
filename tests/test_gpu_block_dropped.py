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


@pytest.mark.parametrize("c", WIDTHS)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("act,post", [("silu", True), ("silu", False), ("sigmoid", True), ("sigmoid", False)])
def test_gradients(c, dtype, act, post):
    # without a norm of its own y may be anything where it is dropped; under one it enters the row's sum
    n, keep, _, d = _inputs(c, dtype, ("gate",) if post else ("gate", "y"))
    (wp, rp), (ws, rs), (wn, rn) = (T._vec(s, c, "f32") for s in (81, 82, 83))
    if not post:
        wp = rp = None
    (x, rx), (y, ry), (z, rz), (go, rgo), (gn, rgn) = (d[k] for k in ("x", "y", "gate", "gout", "gnorm"))
    g = fx.block_join_bwd(go, gn, x, y, gate=z, act=act, post_weight=wp, scale=ws, next_weight=wn, eps=EPS, p=P, seed=SEED, offset=OFFSET)
    want = R.join_grad(rgo, rgn, rx, ry, rz, act, rp, rs, rn, EPS, keep)
    kk = T._k(c) + (2 * np.abs(rz) + 16) * U
    E, Et = T._norm_grad_bound(np.zeros_like(ry), rgn, rx, rn, EPS)
    D, ED = want["x"], U * np.abs(want["x"]) + E
    R.check(T._f64(g["x"]), D, ED, dtype, "x")
    T._sum_check(T._f64(g["next"]), want["next"], Et, "f32", "next")
    yr = ry if rp is None else R.norm(ry, rp, EPS)
    a, da = R.act(rz, act)
    s, t = R.sigmoid(rz), R.sigmoid(-rz)
    da_size = s * t if act == "sigmoid" else s * (1 + np.abs(rz) * t)
    T._sum_check(T._f64(g["scale"]), want["scale"], np.abs(keep * yr * a) * ED + kk * np.abs(want["scale"]), "f32", "scale")
    R.check(T._f64(g["gate"]), want["gate"], np.abs(keep * rs * yr) * (np.abs(da) * ED + kk * np.abs(D) * da_size), dtype, "gate")
    u = D * keep * rs * a
    Eu = np.abs(keep * rs * a) * ED + kk * np.abs(u)
    if post:
        Ey, Ep = T._norm_grad_bound(Eu, u, ry, rp, EPS)
        T._sum_check(T._f64(g["post"]), want["post"], Ep, "f32", "post")
        R.check(T._f64(g["y"]), want["y"], Ey, dtype, "y")
    else:
        R.check(T._f64(g["y"]), want["y"], Eu, dtype, "y")


@pytest.mark.parametrize("c", [45, 64, 520])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinities_under_a_norm_of_their_own(c, dtype):
    """A row whose y has infinities has a norm of zeros but where they lie.  Where they are dropped the row adds nothing to the
    vectors' gradients and has none of the gate; y's is zero but where y is infinite, where the norm has no derivative."""
    n, keep, at, d = _inputs(c, dtype, ())
    y, ry = d["y"]
    bad = torch.from_numpy(at).cuda()
    y[bad] = float("inf")
    rows = at.any(1)
    assert rows.any() and not rows.all()
    (wp, rp), (ws, rs), (wn, _) = (T._vec(s, c, "f32") for s in (81, 82, 83))
    x, z, go = d["x"][0], d["gate"][0], d["gout"][0]
    kw = dict(gate=z, act="silu", post_weight=wp, scale=ws, eps=EPS, p=P, seed=SEED, offset=OFFSET)
    out, norm = fx.block_join_fwd(x, y, next_weight=wn, **kw)
    spoilt = torch.from_numpy(rows).cuda()
    assert torch.equal(out[spoilt], x[spoilt]) and torch.isfinite(norm).all()
    g = fx.block_join_bwd(go, None, None, y, **kw)
    assert not g["gate"][spoilt].any() and torch.isfinite(g["gate"]).all()
    assert torch.isnan(g["y"][bad]).all() and not g["y"][spoilt[:, None] & ~bad].any()
    ok = ~rows
    rz, rgo = d["gate"][1][ok], d["gout"][1][ok]
    want = R.join_grad(rgo, None, None, ry[ok], rz, "silu", rp, rs, None, EPS, keep[ok])
    kk = T._k(c) + (2 * np.abs(rz) + 16) * U
    a = R.act(rz, "silu")[0]
    u = rgo * keep[ok] * rs * a
    T._sum_check(T._f64(g["scale"]), want["scale"], (kk + U) * np.abs(want["scale"]), "f32", "scale")
    T._sum_check(T._f64(g["post"]), want["post"], T._norm_grad_bound((kk + U) * np.abs(u), u, ry[ok], rp, EPS)[1], "f32", "post")
