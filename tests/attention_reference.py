"""Attention, its gradients and the cache from their definitions in 64 bits on the CPU (numpy, one sequence and head at a
time), with bounds on what the kernels' arithmetic may be off by.

u = 2^-24 is fp32's half unit, r the storage type's (tests' inputs are values of that type, so products of two are exact in
fp32, or off by u for fp32 inputs).  A score is a sum of dim products in some order of fp32 additions, off by at most
(dim + 2) u scale sum_d |q_d k_d| =: e; its exponential adds (|x| + 4) u of itself, x the argument in base 2, and is rounded to r
where it meets 16-bit values; an exponential below the least normal number, 2^-126, may come as zero.  Everything else is linear in the weights and is bounded by the same sum over sizes."""
import numpy as np

U = 2.0 ** -24
HALF = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
FLUSH = 2.0 ** -126
LEAST = {"f32": 0.0, "f16": 2.0 ** -25, "bf16": 2.0 ** -134}


def seen_by(nq, nk, causal):
    i, j = np.arange(nq)[:, None], np.arange(nk)[None, :]
    return (nq - i <= nk - j) if causal else np.ones((nq, nk), bool)


def _weights(q, k, scale, seen):
    """Probabilities, lse and the relative error of every probability, of one head."""
    s = np.where(seen, scale * (q @ k.T), -np.inf)
    e = np.where(seen, (q.shape[1] + 2) * U * abs(scale) * (np.abs(q) @ np.abs(k).T), 0.0)
    top = np.where(seen.any(1, keepdims=True), s.max(1, keepdims=True, initial=-np.inf), 0.0)
    x = np.exp(s - top)
    total = x.sum(1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = (top + np.log(total))[:, 0]
    p = x / np.where(total > 0, total, 1)
    # the argument's rounding, that of its two terms, the exponential; the row's largest for the sum they are divided by
    size = np.where(seen, np.abs(np.where(seen, s, 0)) + np.abs(top), 0.0) * 1.45
    rel = e + (2 * size + 8) * U
    worst = rel.max(1, keepdims=True, initial=0.0) + (k.shape[0] / 8 + 16) * U
    return p, lse, rel + worst, worst[:, 0]


def attention(q, k, v, bq, bk, causal, scale, dtype):
    """out, lse and bounds of both; q [rows, heads, dim], k, v [rows, kv_heads, dim] in 64 bits."""
    g = q.shape[1] // k.shape[1]
    out, lse = np.zeros_like(q), np.full((q.shape[1], q.shape[0]), -np.inf)
    bo, bl = np.zeros_like(q), np.zeros_like(lse)
    r = 0.0 if dtype == "f32" else HALF[dtype]
    for a0, a1, b0, b1 in zip(bq[:-1], bq[1:], bk[:-1], bk[1:]):
        if a1 == a0 or b1 == b0:
            continue
        seen = seen_by(a1 - a0, b1 - b0, causal)
        for h in range(q.shape[1]):
            kk, vv = k[b0:b1, h // g], v[b0:b1, h // g]
            p, l, rel, worst = _weights(q[a0:a1, h], kk, scale, seen)
            out[a0:a1, h], lse[h, a0:a1] = p @ vv, l
            bo[a0:a1, h] = (p * (rel + r + ((b1 - b0) / 8 + 8) * U)) @ np.abs(vv) + (LEAST[dtype] * 256 + FLUSH) * np.abs(vv).sum(0)
            bl[h, a0:a1] = np.where(np.isfinite(l), worst + 8 * U * (np.abs(np.where(np.isfinite(l), l, 0)) + 1), 0)
    return out, lse, bo, bl


def attention_grad(q, k, v, go, bq, bk, causal, scale, dtype, glse=None):
    """gq, gk, gv and bounds of the three."""
    g = q.shape[1] // k.shape[1]
    gq, gk, gv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    eq, ek, ev = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    r = 0.0 if dtype == "f32" else HALF[dtype]
    for a0, a1, b0, b1 in zip(bq[:-1], bq[1:], bk[:-1], bk[1:]):
        if a1 == a0 or b1 == b0:
            continue
        seen = seen_by(a1 - a0, b1 - b0, causal)
        add = ((max(a1 - a0, b1 - b0)) * g / 8 + 16) * U
        for h in range(q.shape[1]):
            qq, kk, vv, gg = q[a0:a1, h], k[b0:b1, h // g], v[b0:b1, h // g], go[a0:a1, h]
            p, l, rel, _ = _weights(qq, kk, scale, seen)
            # recomputed from lse, whose size's rounding it takes along
            rel = rel + 4 * U * (np.abs(np.where(np.isfinite(l), l, 0)) + 1)[:, None]
            dp = gg @ vv.T
            edp = (q.shape[2] + 2) * U * (np.abs(gg) @ np.abs(vv).T)
            delta = (p * dp).sum(1, keepdims=True)
            # out is rounded to its type before its product with gout; its weights were too
            size = np.abs(gg) * (p @ np.abs(vv))
            edelta = ((HALF[dtype] + 2 * r + rel.max(1, keepdims=True) + add) * size).sum(1, keepdims=True) + (p * edp).sum(1, keepdims=True)
            more = 0.0 if glse is None else glse[h, a0:a1][:, None]
            inner = dp - delta + more
            ds = p * inner
            eds = p * (edp + edelta + 4 * U * (np.abs(dp) + np.abs(delta) + np.abs(more))) + (rel + r) * np.abs(ds) + LEAST[dtype] + FLUSH * np.abs(inner)
            ep = (rel + r) * p + LEAST[dtype] + FLUSH
            j = h // g
            gq[a0:a1, h], eq[a0:a1, h] = scale * (ds @ kk), abs(scale) * ((eds + add * np.abs(ds)) @ np.abs(kk))
            gk[b0:b1, j] += scale * (ds.T @ qq)
            ek[b0:b1, j] += abs(scale) * ((eds + add * np.abs(ds)).T @ np.abs(qq))
            gv[b0:b1, j] += p.T @ gg
            ev[b0:b1, j] += (ep + add * p).T @ np.abs(gg)
    return gq, gk, gv, eq, ek, ev


def check(got, ref, bound, dtype, what=""):
    """got against ref: off by the bound and one rounding to the storage type at most; infinities and NaN where ref has them."""
    assert got.shape == ref.shape, what
    odd = ~np.isfinite(ref)
    assert np.array_equal(got[odd], ref[odd], equal_nan=True), f"{what}: infinities or NaN differ"
    off, half = np.abs(got - ref)[~odd], HALF[dtype]
    allowed = (bound + half * (np.abs(np.where(odd, 0, ref)) + bound) + LEAST[dtype] + 1e-37)[~odd]
    bad = ~(off <= allowed)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, {np.nanmax(np.where(bad, off / allowed, 0)):.2f} times the bound, NaN: {np.isnan(off).sum()}"


def exponents(x):
    """Exponents (plus 127) of rows in a cache of 8 bits: the least e >= -127 with no finite value over 448 2^e."""
    top = np.abs(np.where(np.isfinite(x), x, 0)).max(-1)
    out = np.zeros(top.shape, np.int64)
    while (more := top > 448.0 * np.exp2(out - 127.0)).any():
        out[more] += 1
    return out


def quantised(x):
    """Values that a cache of 8 bits holds of rows."""
    grid = np.array(sorted({(m / 8 if e == 0 else 1 + m / 8) * 2.0 ** (max(e, 1) - 7) for e in range(16) for m in range(8) if (e, m) != (15, 7)}))
    e = exponents(x)[..., None] - 127
    u = np.abs(np.where(np.isfinite(x), x, 0)) * 2.0 ** -e.astype(float)
    hi = np.searchsorted(grid, u).clip(max=len(grid) - 1)
    lo = np.maximum(hi - 1, 0)
    up = (grid[hi] - u < u - grid[lo]) | ((grid[hi] - u == u - grid[lo]) & (hi % 2 == 0))      # grid[i] has code i: ties go to even codes
    y = np.where(u == grid[hi], u, np.where(up, grid[hi], grid[lo])) * 2.0 ** e.astype(float)
    return np.where(np.isfinite(x), np.copysign(y, x), np.nan)
