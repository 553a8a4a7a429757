"""The operators around the convolution, from their definitions in 64 bits on the CPU (numpy, one row after the other),
with bounds on what fp32 arithmetic may be off by.

A sigmoid computed in fp32 is off by (2 |z| + 8) u of its size, u = 2^-24: the argument's rounding (|z| u), and a few
units for the exponential, the sum, the reciprocal and the product.  The recurrence's bound follows the recurrence
itself, E_t = f E_(t-1) + c u (|f h_(t-1)| + |g x|) with c = 2 |z| + 16: a step's own roundings, the gate's, and the
product of gates that joins runs of rows.  Sums over n values are bounded by their size times (n/8 + 8) u in any order
with at least eight independent parts."""
import numpy as np

U = 2.0 ** -24
# half a unit in the last place, relative; and half the smallest subnormal number
ROUNDING = {"f32": (0.0, 0.0), "f16": (2.0 ** -11, 2.0 ** -25), "bf16": (2.0 ** -8, 2.0 ** -134)}


def sigmoid(z):
    e = np.exp(-np.abs(z))
    return np.where(z > 0, 1 / (1 + e), e / (1 + e))


def check(got, ref, bound, dtype, what=""):
    """got (float64 of the stored values) against ref, off by the bound and one rounding to the storage type at most."""
    rel, least = ROUNDING[dtype]
    off = np.abs(got - ref)
    allowed = bound + rel * (np.abs(ref) + bound) + least + 1e-37
    bad = ~(off <= allowed)
    assert got.shape == ref.shape and not bad.any(), \
        f"{what}: {bad.sum()} of {bad.size}, first at {np.argwhere(bad)[0]}: {got[tuple(np.argwhere(bad)[0])]} for {ref[tuple(np.argwhere(bad)[0])]}, " \
        f"{(off / allowed)[bad].max():.2f} times the bound"


def scan(x, gate, bounds, h0=None, reverse=False):
    """h, last and the bounds of both."""
    f, g, c = sigmoid(gate), sigmoid(-gate), 2 * np.abs(gate) + 16
    h, E = np.zeros_like(x), np.zeros_like(x)
    n_seq = len(bounds) - 1
    last = np.zeros((n_seq, x.shape[1])) if h0 is None else h0.copy()
    last_E = np.zeros_like(last)
    for s in range(n_seq):
        rows = range(bounds[s], bounds[s + 1])
        v, e = last[s], last_E[s]
        for t in (reversed(rows) if reverse else rows):
            e = f[t] * e + c[t] * U * (np.abs(f[t] * v) + np.abs(g[t] * x[t]))
            v = f[t] * v + g[t] * x[t]
            h[t], E[t] = v, e
        last[s], last_E[s] = v, e
    return h, last, E, last_E


def scan_grad(x, gate, h, gh, bounds, h0=None, glast=None, reverse=False):
    """gx, ggate, gh0 and the bounds of the three; h is taken as given."""
    f, g, c = sigmoid(gate), sigmoid(-gate), 2 * np.abs(gate) + 16
    gx, gz, Ex, Ez = (np.zeros_like(x) for _ in range(4))
    n_seq = len(bounds) - 1
    m0 = np.zeros((n_seq, x.shape[1])) if glast is None else glast.copy()
    E0 = np.zeros_like(m0)
    for s in range(n_seq):
        a, b = bounds[s], bounds[s + 1]
        rows = list(range(a, b))[::-1] if reverse else list(range(a, b))
        m, e = m0[s], E0[s]
        for k in range(len(rows) - 1, -1, -1):
            t = rows[k]
            before = h[rows[k - 1]] if k else (np.zeros(x.shape[1]) if h0 is None else h0[s])
            lam, el = gh[t] + m, e + U * np.abs(gh[t] + m)
            gx[t], gz[t] = g[t] * lam, lam * (before - x[t]) * f[t] * g[t]
            Ex[t] = g[t] * el + c[t] * U * np.abs(gx[t])
            Ez[t] = np.abs(before - x[t]) * f[t] * g[t] * el + 2 * c[t] * U * np.abs(gz[t])
            m, e = f[t] * lam, f[t] * el + c[t] * U * (np.abs(f[t] * gh[t]) + np.abs(f[t] * m))
        m0[s], E0[s] = m, e
    return gx, gz, m0, Ex, Ez, E0


def keep_mask(rows, c, p, seed, offset):
    """True where dropout keeps a value, by Python's whole numbers."""
    t = int(p * 65536 + 0.5)
    out = np.zeros((rows, c), bool)
    low = 0xFFFFFFFF
    for r in range(rows):
        for q in range((c + 7) // 8):
            w, k = [q, r, offset & low, (offset >> 32) & low], [seed & low, (seed >> 32) & low]
            for _ in range(7):
                a, b = w[0] * 0xD2511F53, w[2] * 0xCD9E8D57
                w = [(b >> 32) ^ w[1] ^ k[0], b & low, (a >> 32) ^ w[3] ^ k[1], a & low]
                k = [(k[0] + 0x9E3779B9) & low, (k[1] + 0xBB67AE85) & low]
            for e in range(min(8, c - 8 * q)):
                out[r, 8 * q + e] = (w[e >> 1] >> (16 * (e & 1)) & 0xFFFF) >= t
    return out


def drop_factor(p):
    t = int(p * 65536 + 0.5)
    return 65536 / (65536 - t) if t < 65536 else 0.0


def norm(x, w, eps):
    return x / np.sqrt((x * x).mean(1, keepdims=True) + eps) * w


def norm_grad(g, x, w, eps):
    r = 1 / np.sqrt((x * x).mean(1, keepdims=True) + eps)
    xh = x * r
    return r * (g * w - xh * (g * w * xh).mean(1, keepdims=True)), g * xh


def act(z, kind):
    s, t = sigmoid(z), sigmoid(-z)
    return (s, s * t) if kind == "sigmoid" else (z * s, s * (1 + z * t))


def join(x, y, gate=None, kind="silu", post=None, scale=None, nxt=None, eps=1e-6, keep=None):
    """out, norm (None without nxt); keep: what drop multiplies by."""
    r = y if post is None else norm(y, post, eps)
    a = 1.0 if gate is None else act(gate, kind)[0]
    out = x + (1.0 if scale is None else scale) * (r * a * (1.0 if keep is None else keep))
    return out, None if nxt is None else norm(out, nxt, eps)


def join_grad(gout, gnorm, out, y, gate=None, kind="silu", post=None, scale=None, nxt=None, eps=1e-6, keep=None):
    """Gradients by name; those of the vectors as terms [rows, C] whose sum over the rows they are."""
    D = np.zeros_like(y) if gout is None else gout.copy()
    g = {}
    if nxt is not None:
        g["next"] = np.zeros_like(y)
        if gnorm is not None:
            gn, g["next"] = norm_grad(gnorm, out, nxt, eps)
            D = D + gn
    g["x"] = D
    r = y if post is None else norm(y, post, eps)
    a, da = (1.0, 0.0) if gate is None else act(gate, kind)
    t = D * (1.0 if keep is None else keep)
    if scale is not None:
        g["scale"] = t * r * a
        t = t * scale
    if gate is not None:
        g["gate"] = t * r * da
    t = t * a
    if post is not None:
        t, g["post"] = norm_grad(t, y, post, eps)
    g["y"] = t
    return g
