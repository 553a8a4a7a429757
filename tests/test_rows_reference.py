"""The oracle of the operators around the convolution against differences of its own forward formulas, and dropout's
generator by its shares (equal, and no dependence on the rows' number)."""
import numpy as np
import pytest

import rows_reference as R


def _difference(fn, args, k, d, eps=1e-6):
    up, down = list(args), list(args)
    up[k], down[k] = args[k] + eps * d, args[k] - eps * d
    return (fn(*up) - fn(*down)) / (2 * eps)


@pytest.mark.parametrize("reverse", [False, True])
def test_scan_gradients_are_the_differences(reverse):
    rng = np.random.default_rng(3)
    bounds = [0, 4, 4, 5, 23]
    x, z, gh = (rng.standard_normal((23, 3)) for _ in range(3))
    h0, gl = rng.standard_normal((4, 3)), rng.standard_normal((4, 3))

    def loss(x, z, h0):
        h, last = R.scan(x, z, bounds, h0, reverse)[:2]
        return (h * gh).sum() + (last * gl).sum()

    h = R.scan(x, z, bounds, h0, reverse)[0]
    grads = R.scan_grad(x, z, h, gh, bounds, h0, gl, reverse)[:3]
    for k, g in enumerate(grads):
        d = rng.standard_normal(g.shape)
        assert abs(_difference(loss, (x, z, h0), k, d) - (g * d).sum()) <= 1e-7 * np.abs(g * d).sum()


@pytest.mark.parametrize("kind", ["silu", "sigmoid"])
def test_join_gradients_are_the_differences(kind):
    rng = np.random.default_rng(4)
    x, y, z, go, gn = (rng.standard_normal((9, 5)) for _ in range(5))
    post, scale, nxt = (rng.standard_normal(5) for _ in range(3))
    keep = R.keep_mask(9, 5, 0.3, 11, 12) * R.drop_factor(0.3)

    def loss(x, y, z, post, scale, nxt):
        out, n = R.join(x, y, z, kind, post, scale, nxt, 1e-3, keep)
        return (out * go).sum() + (n * gn).sum()

    out = R.join(x, y, z, kind, post, scale, nxt, 1e-3, keep)[0]
    g = R.join_grad(go, gn, out, y, z, kind, post, scale, nxt, 1e-3, keep)
    for k, name in enumerate(("x", "y", "gate", "post", "scale", "next")):
        gr = g[name] if k < 3 else g[name].sum(0)
        d = rng.standard_normal(gr.shape)
        assert abs(_difference(loss, (x, y, z, post, scale, nxt), k, d) - (gr * d).sum()) <= 1e-7 * np.abs(gr * d).sum()


def test_mask_shares_and_independence():
    n, c, p = 400, 40, 0.25
    m = R.keep_mask(n, c, p, 0x123456789ABCDEF0, 77)
    share = m.mean()
    assert abs(share - 0.75) <= 5 * np.sqrt(0.75 * 0.25 / m.size)               # five standard deviations
    assert np.abs(m.mean(0) - 0.75).max() <= 5 * np.sqrt(0.75 * 0.25 / n)
    other = R.keep_mask(n, c, p, 0x123456789ABCDEF0, 78)
    assert abs((m & other).mean() - 0.75 ** 2) <= 5 * np.sqrt(0.5625 * 0.4375 / m.size)
    # a value's number depends on its row and channel alone
    assert np.array_equal(R.keep_mask(5, 13, p, 0x123456789ABCDEF0, 77), m[:5, :13])


def test_a_planted_mistake_is_found():
    rng = np.random.default_rng(5)
    x, z = rng.standard_normal((30, 4)), rng.standard_normal((30, 4))
    h, last, E, _ = R.scan(x, z, [0, 30])
    wrong = R.scan(x, np.where(np.arange(30)[:, None] == 17, z + 1e-3, z), [0, 30])[0]
    R.check(h, h, E, "f32")
    with pytest.raises(AssertionError):
        R.check(wrong, h, E, "f32")
