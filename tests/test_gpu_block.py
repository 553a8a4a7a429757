"""GPU parity of a block's norms, join and dropout: outputs and gradients against the formulas in 64 bits, at widths
around a piece (8 channels), a wave (512) and a workgroup a row, every type, column ranges of wider tensors, inputs
left out, in place; masks bit for bit."""
import itertools

import numpy as np
import pytest
import torch

import gpu_common as H
import paper_2407_01781_amd as fx
import rows_reference as R

pytestmark = pytest.mark.gpu
U = R.U


def _draw(seed, n, c, dtype, packed=False, std=1.0, mean=0.0):
    rng = np.random.default_rng(seed)
    v = torch.from_numpy((rng.standard_normal((n, c)) * std + mean).astype(np.float32)).to(H.TORCH_DT[dtype])
    if packed:
        wide = torch.full((n, c + 4), 7.0, dtype=v.dtype, device="cuda")
        wide[:, 1:c + 1] = v.cuda()
        return wide[:, 1:c + 1], v.double().numpy()
    return v.cuda(), v.double().numpy()


def _vec(seed, c, dtype, std=0.3, mean=1.0):
    d, v = _draw(seed, 1, c, dtype, False, std, mean)
    return d.reshape(-1).contiguous(), v.reshape(-1)


def _f64(t):
    return t.double().cpu().numpy()


# Bounds: a row's sum of C squares is off by (C / 8 + 8) units, its root and quotient by 8 more; k(C) covers a product
# with them.  What follows is off by what its factors are off by.
def _k(c):
    return (c / 8 + 24) * U


def _norm_grad_bound(Eg, g, x, w, eps):
    r = 1 / np.sqrt((x * x).mean(1, keepdims=True) + eps)
    xh = np.abs(x * r)
    size = lambda t: r * (np.abs(t * w) + xh * (np.abs(t * w) * xh).mean(1, keepdims=True))
    return size(Eg) + 3 * _k(x.shape[1]) * size(g), xh * Eg + 2 * _k(x.shape[1]) * np.abs(g) * xh


def _sum_check(got, terms, E, dtype, what):
    n = terms.shape[0]
    R.check(got, terms.sum(0), E.sum(0) + (n / 8 + 8) * U * np.abs(terms).sum(0), dtype, what)


WIDTHS = [1, 3, 7, 8, 9, 16, 45, 64, 100, 256, 511, 512, 513, 1000, 2048, 4095, 4096]


@pytest.mark.parametrize("c", WIDTHS)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_norm(c, dtype):
    n = 1 if c == 16 else 37 if c > 600 else 333
    packed, vdt = c % 2 == 1, dtype if c % 3 else "f32"
    x, rx = _draw(1, n, c, dtype, packed, std=2.0)
    g, rg = _draw(2, n, c, dtype, packed)
    w, rw = _vec(3, c, vdt)
    out = H.nan_filled((n, c), x.dtype)
    ref = R.norm(rx, rw, 1e-5)
    R.check(_f64(fx.rms_norm_fwd(x, w, 1e-5, out=out)), ref, _k(c) * np.abs(ref), dtype, "norm")
    gx, gw = fx.rms_norm_bwd(g, x, w, 1e-5)
    want, terms = R.norm_grad(rg, rx, rw, 1e-5)
    Ex, Ew = _norm_grad_bound(np.zeros_like(rg), rg, rx, rw, 1e-5)
    R.check(_f64(gx), want, Ex, dtype, "gx")
    _sum_check(_f64(gw), terms, Ew, vdt, "gweight")
    again = fx.rms_norm_bwd(g, x, w, 1e-5)
    assert torch.equal(gx, again[0]) and torch.equal(gw, again[1])
    plain = fx.rms_norm_fwd(x, None, 1e-5)
    R.check(_f64(plain), R.norm(rx, 1.0, 1e-5), _k(c) * np.abs(R.norm(rx, 1.0, 1e-5)), dtype, "without a weight")
    assert fx.rms_norm_bwd(g, x, None, 1e-5)[1] is None
    y = x.clone()
    assert torch.equal(fx.rms_norm_fwd(y, w, 1e-5, out=y), out)                  # in place


def test_norm_over_many_rows():
    n, c = 70_001, 40
    x, rx = _draw(4, n, c, "bf16")
    g, rg = _draw(5, n, c, "bf16")
    w, rw = _vec(6, c, "f32")
    ref = R.norm(rx, rw, 1e-6)
    R.check(_f64(fx.rms_norm_fwd(x, w)), ref, _k(c) * np.abs(ref), "bf16")
    gx, gw = fx.rms_norm_bwd(g, x, w)
    want, terms = R.norm_grad(rg, rx, rw, 1e-6)
    Ex, Ew = _norm_grad_bound(np.zeros_like(rg), rg, rx, rw, 1e-6)
    R.check(_f64(gx), want, Ex, "bf16")
    _sum_check(_f64(gw), terms, Ew, "f32", "gweight")


def test_rows_of_zeros_and_no_rows():
    x = torch.zeros((5, 24), device="cuda")
    w = torch.ones(24, device="cuda")
    assert torch.equal(fx.rms_norm_fwd(x, w), x)
    gx, gw = fx.rms_norm_bwd(torch.ones_like(x), x, w, 1e-6)
    assert torch.isfinite(gx).all() and torch.equal(gw, torch.zeros_like(w))
    e = torch.empty((0, 24), device="cuda")
    assert fx.rms_norm_fwd(e, w).shape == (0, 24)
    assert torch.equal(fx.rms_norm_bwd(e, e, w)[1], torch.zeros_like(w))
    assert fx.dropout(e, 0.5, 1, 2).shape == (0, 24)
    out, n = fx.block_join_fwd(e, e, gate=e, post_weight=w, scale=w, next_weight=w)
    assert out.shape == n.shape == (0, 24)
    g = fx.block_join_bwd(e, e, out, e, gate=e, post_weight=w, scale=w, next_weight=w)
    assert all(torch.equal(g[k], torch.zeros_like(w)) for k in ("post", "scale", "next"))


def _join_case(n, c, dtype, vdt, packed, gate, act, post, scale, nxt, p, give=(True, True), eps=1e-5):
    x, rx = _draw(11, n, c, dtype, packed, std=1.5)
    y, ry = _draw(12, n, c, dtype, packed, std=3.0)
    z, rz = _draw(13, n, c, dtype, packed, std=1.5) if gate else (None, None)
    go, rgo = _draw(14, n, c, dtype, packed)
    gn, rgn = _draw(15, n, c, dtype, packed)
    wp, rwp = _vec(16, c, vdt) if post else (None, None)
    ws, rws = _vec(17, c, vdt) if scale else (None, None)
    wn, rwn = _vec(18, c, vdt) if nxt else (None, None)
    seed, offset = 0xFEDCBA9876543210, (5 << 32) + 99
    keep = R.keep_mask(n, c, p, seed, offset) * R.drop_factor(p)
    kw = dict(gate=z, act=act, post_weight=wp, scale=ws, next_weight=wn, eps=eps, p=p, seed=seed, offset=offset)
    out, norm = fx.block_join_fwd(x, y, **kw)
    ref, rnorm = R.join(rx, ry, rz, act, rwp, rws, rwn, eps, keep)
    zz = 0.0 if rz is None else 2 * np.abs(rz) + 16
    Eo = (_k(c) + zz * U) * np.abs(ref - rx) + U * np.abs(ref)
    R.check(_f64(out), ref, Eo, dtype, "out")
    if nxt:
        r = 1 / np.sqrt((ref * ref).mean(1, keepdims=True) + eps)
        En = np.abs(rwn) * r * (Eo + np.abs(ref) * (_k(c) + r * np.sqrt((Eo * Eo).mean(1, keepdims=True))))
        R.check(_f64(norm), rnorm, En, dtype, "norm")
    else:
        assert norm is None
    if not give[0]:
        go = rgo = None
    if not (give[1] and nxt):
        gn = rgn = None
    g = fx.block_join_bwd(go, gn, out, y, **kw)
    ro = _f64(out)
    want = R.join_grad(rgo, rgn, ro, ry, rz, act, rwp, rws, rwn, eps, keep)
    one = np.ones_like(ry)
    D, ED = want["x"], U * np.abs(want["x"])
    if rgn is not None:
        E, Et = _norm_grad_bound(0 * one, rgn, ro, rwn, eps)
        ED = ED + E
        _sum_check(_f64(g["next"]), want["next"], Et, vdt, "next")
    elif nxt:
        assert not g["next"].any()
    R.check(_f64(g["x"]), D, ED, dtype, "x")
    yr = ry if rwp is None else R.norm(ry, rwp, eps)
    a, da, da_size = one, 0 * one, 0 * one
    if gate:
        a, da = R.act(rz, act)
        s, t = R.sigmoid(rz), R.sigmoid(-rz)
        da_size = s * t if act == "sigmoid" else s * (1 + np.abs(rz) * t)
    kk = _k(c) + zz * U
    sc = one if rws is None else rws * one
    if scale:
        co = keep * yr * a
        _sum_check(_f64(g["scale"]), want["scale"], np.abs(co) * ED + kk * np.abs(want["scale"]), vdt, "scale")
    if gate:
        co = keep * sc * yr
        R.check(_f64(g["gate"]), want["gate"], np.abs(co) * (np.abs(da) * ED + kk * np.abs(D) * da_size), dtype, "gate")
    u = D * keep * sc * a
    Eu = np.abs(keep * sc * a) * ED + kk * np.abs(u)
    if post:
        Ey, Ep = _norm_grad_bound(Eu, u, ry, rwp, eps)
        _sum_check(_f64(g["post"]), want["post"], Ep, vdt, "post")
        R.check(_f64(g["y"]), want["y"], Ey, dtype, "y")
    else:
        R.check(_f64(g["y"]), want["y"], Eu, dtype, "y")
    for k, on in (("gate", gate), ("post", post), ("scale", scale), ("next", nxt)):
        assert (g[k] is not None) == on
    again = fx.block_join_bwd(go, gn, out, y, **kw)
    assert all(g[k] is None or torch.equal(g[k], again[k]) for k in g)
    # in place: the sum where x lies
    x2 = x.clone()
    same, n2 = fx.block_join_fwd(x2, y, out=x2, **kw)
    assert torch.equal(same, out) and (norm is None or torch.equal(n2, norm))


@pytest.mark.parametrize("gate,post,scale,nxt", list(itertools.product([False, True], repeat=4)))
@pytest.mark.parametrize("act,p", [("silu", 0.0), ("sigmoid", 0.3)])
def test_join_with_inputs_left_out(gate, post, scale, nxt, act, p):
    _join_case(61, 45, "f32", "f32", False, gate, act, post, scale, nxt, p)


@pytest.mark.parametrize("c", WIDTHS)
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_join_widths(c, dtype):
    n = 1 if c == 16 else 9 if c > 600 else 77
    _join_case(n, c, dtype, dtype if c % 3 else "f32", c % 2 == 1, True, "silu", True, True, True, 0.2)


@pytest.mark.parametrize("give", [(True, False), (False, True)])
def test_join_with_the_gradient_of_one_output(give):
    _join_case(50, 64, "bf16", "f32", False, True, "silu", True, True, True, 0.1, give)


def test_join_over_many_rows():
    _join_case(9_001, 24, "bf16", "f32", False, True, "silu", True, True, True, 0.1)


def test_join_gradient_is_the_difference():
    """Derivatives along a direction in y and in the gate, from fp32 outputs at a step of 2^-6 either side: third
    derivatives and sums of 2e3 terms rounded to 2^-24 stay below half a per cent."""
    n, c = 64, 32
    (x, _), (y, _), (z, _), (go, _), (gn, _), (d, _) = (_draw(s, n, c, "f32") for s in range(21, 27))
    (wp, _), (ws, _), (wn, _) = (_vec(s, c, "f32") for s in (27, 28, 29))
    kw = dict(act="silu", post_weight=wp, scale=ws, next_weight=wn, p=0.2, seed=3, offset=4)

    def loss(y, z):
        o, m = fx.block_join_fwd(x, y, gate=z, **kw)
        return float((o.double() * go.double()).sum() + (m.double() * gn.double()).sum())

    out = fx.block_join_fwd(x, y, gate=z, **kw)[0]
    g = fx.block_join_bwd(go, gn, out, y, gate=z, **kw)
    eps = 2.0 ** -6
    for name, (a, b) in (("y", (eps, 0.0)), ("gate", (0.0, eps))):
        num = (loss(y + a * d, z + b * d) - loss(y - a * d, z - b * d)) / (2 * eps)
        assert abs(num - float((g[name].double() * d.double()).sum())) <= 5e-3 * float((g[name].double() * d.double()).norm())


@pytest.mark.parametrize("c", [1, 5, 8, 45, 64, 520, 1030])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_dropout(c, dtype, p):
    n = 19 if c > 500 else 150
    x, rx = _draw(31, n, c, dtype, packed=c % 2 == 1)
    res, rres = _draw(32, n, c, dtype, packed=c % 2 == 1)
    seed, offset = 2 ** 64 - 3, 2 ** 40 + 17
    m = R.keep_mask(n, c, p, seed, offset)
    ref = np.where(m, rx * R.drop_factor(p), 0.0)
    got = fx.dropout(x, p, seed, offset)
    R.check(_f64(got), ref, U * np.abs(ref), dtype)
    assert np.array_equal(_f64(got) != 0, m & (rx != 0))
    R.check(_f64(fx.dropout(x, p, seed, offset, residual=res)), ref + rres, 2 * U * (np.abs(ref) + np.abs(rres)), dtype)
    y = res.clone()
    assert torch.equal(fx.dropout(x, p, seed, offset, residual=y, out=y), fx.dropout(x, p, seed, offset, residual=res))
    y = x.clone()
    assert torch.equal(fx.dropout(y, p, seed, offset, out=y), got)


def test_dropped_values_leave_nothing():
    x = torch.full((200, 24), float("nan"), device="cuda")
    x[::2] = float("inf")
    m = torch.from_numpy(R.keep_mask(200, 24, 0.5, 5, 6)).cuda()
    y = fx.dropout(x, 0.5, 5, 6)
    assert not y[~m].any()
    assert torch.isinf(y[::2][m[::2]]).all() and torch.isnan(y[1::2][m[1::2]]).all()
    # a dropped value's gradient is zero whatever the value is; the block's too
    out = fx.block_join_fwd(torch.zeros_like(x), x, p=0.5, seed=5, offset=6)[0]
    assert torch.equal(torch.isfinite(out), ~m) and not out[~m].any()
    g = fx.block_join_bwd(torch.ones_like(x), None, None, x, p=0.5, seed=5, offset=6)
    assert torch.equal(g["y"], m.float() * 2)


def test_offset_from_the_device_and_graph_replays():
    """A captured block whose owner raises the offset between replays: every replay equal to the call made directly."""
    n, c = 3_000, 48
    (x, _), (y, _), (z, _) = (_draw(s, n, c, "bf16") for s in (41, 42, 43))
    (wp, _), (ws, _), (wn, _) = (_vec(s, c, "f32") for s in (44, 45, 46))
    seqs = fx.build_sequences([[0, 1_000], [1_000, n]])
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    fx.use_torch_allocator(True)
    try:
        def block(d_offset, offset):
            h, _ = fx.gated_scan_fwd(seqs, y, z)
            out, norm = fx.block_join_fwd(x, h, gate=z, post_weight=wp, scale=ws, next_weight=wn, p=0.2, seed=9, offset=offset, d_offset=d_offset)
            g = fx.block_join_bwd(norm, out, out, h, gate=z, post_weight=wp, scale=ws, next_weight=wn, p=0.2, seed=9, offset=offset, d_offset=d_offset)
            gx, gz, _ = fx.gated_scan_bwd(seqs, y, z, h, g["y"])
            return [h, out, norm, gx, gz, fx.dropout(gx, 0.1, 9, offset + 1, d_offset=d_offset)] + [t for t in g.values()]

        block(step, 1_000)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = block(step, 1_000)
        for i in range(4):
            step.fill_(i)
            y.copy_(_draw(50 + i, n, c, "bf16")[0])
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, block(None, 1_000 + i)))
        del graph, out
    finally:
        torch.cuda.synchronize()
        import gc
        seqs = None
        gc.collect()
        fx.use_torch_allocator(False)


def test_offsets_beyond_32_bits():
    n, c, ld = 5_000, 64, 500_000
    wide = torch.empty(n * ld, dtype=torch.bfloat16, device="cuda")
    x, y = wide.as_strided((n, c), (ld, 1), 0), wide.as_strided((n, c), (ld, 1), 1_000)
    small = [_draw(s, n, c, "bf16")[0] for s in (61, 62)]
    x.copy_(small[0])
    y.copy_(small[1])
    w = torch.ones(c, device="cuda")
    kw = dict(post_weight=w, next_weight=w, p=0.1, seed=1, offset=2)
    a, b = fx.block_join_fwd(x, y, out=wide.as_strided((n, c), (ld, 1), 2_000), **kw), fx.block_join_fwd(*small, **kw)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    ga, gb = fx.block_join_bwd(x, y, a[0], y, **kw), fx.block_join_bwd(small[0], small[1], b[0], small[1], **kw)
    assert all(ga[k] is None or torch.equal(ga[k], gb[k]) for k in ga)


def test_refusals():
    x = torch.zeros((4, 16), device="cuda")
    w = torch.ones(16, device="cuda")
    with pytest.raises(fx.FxError) as e:
        fx.rms_norm_fwd(torch.zeros((2, 4_097), device="cuda"))
    assert e.value.status == -5
    for eps in (-1e-6, float("inf"), float("nan")):
        with pytest.raises(fx.FxError) as e:
            fx.rms_norm_fwd(x, w, eps)
        assert e.value.status == -1
    for p in (-0.1, 1.1, float("nan")):
        with pytest.raises(fx.FxError) as e:
            fx.dropout(x, p, 1, 2)
        assert e.value.status == -1
    with pytest.raises(fx.FxError):
        fx.rms_norm_fwd(x[:1].expand(4, 16), w)                     # rows on top of each other
    with pytest.raises(fx.FxError):
        fx.block_join_bwd(None, None, x, x, next_weight=w)          # no gradient at all
    with pytest.raises(fx.FxError):
        fx.block_join_bwd(x, x, x, x)                               # the gradient of an output that is not there
    with pytest.raises(fx.FxError):
        fx.block_join_bwd(x, x, None, x, next_weight=w)             # without the output it needs
    with pytest.raises(AssertionError):
        fx.rms_norm_fwd(x, w[:8])
    with pytest.raises(AssertionError):
        fx.block_join_fwd(x, x.half())
    with pytest.raises(AssertionError):
        fx.block_join_fwd(x, x, post_weight=w, scale=w.half())
    with pytest.raises(KeyError):
        fx.block_join_fwd(x, x, gate=x, act="relu")
    assert torch.equal(fx.rms_norm_fwd(x, w), x)
