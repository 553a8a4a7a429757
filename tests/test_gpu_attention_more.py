"""More of attention against the formulas in 64 bits: gradients against differences, gradients that are not asked for, the step with
many heads, many splits and shared pages, many short sequences, every way in which few or many rows are shared out, the same bits from
every call."""
import ctypes as C

import numpy as np
import pytest
import torch

import attention_reference as A
import paper_2407_01781_amd as fx
from paper_2407_01781_amd import binding as B
from test_gpu_attention import _f64, _held, _joff, _tables, draw, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,kv_heads", [(16, 1), (17, 1), (24, 1), (40, 1), (64, 2), (33, 33)])
@pytest.mark.parametrize("dtype,store", [("bf16", "e4m3"), ("f16", "f16"), ("f32", "f32")])
def test_step_with_many_heads(heads, kv_heads, dtype, store):
    rng = np.random.default_rng(heads)
    lens, d, page = [70, 0, 1300], 48, 16
    bounds, jo = _joff(lens)
    table, pages = _tables(rng, lens, page)
    cache = fx.KVCache.empty(pages, page, kv_heads, d, torch.float8_e4m3fn if store == "e4m3" else {"f16": torch.float16, "f32": torch.float32}[store])
    k, k64 = draw(1, bounds[-1], kv_heads, d, dtype)
    v, v64 = draw(2, bounds[-1], kv_heads, d, dtype)
    q, q64 = draw(3, 3, heads, d, dtype, std=2.0)
    fx.cache_write(cache, table, torch.zeros(3, dtype=torch.int32, device="cuda"), k, v, seqs=fx.build_sequences(jo))
    out, lse = fx.attention_step(cache, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), q)
    ro, rl, bo, bl = A.attention(q64, _held(k64, store), _held(v64, store), np.arange(4), bounds, False, d ** -0.5, dtype)
    A.check(_f64(out), ro, bo, dtype, "out")
    A.check(_f64(lse), rl.T, bl.T, "f32", "lse")


@pytest.mark.parametrize("n", [257, 1024, 1025, 5000, 300_000])
@pytest.mark.parametrize("d,store", [(64, "bf16"), (128, "e4m3"), (20, "bf16")])
def test_step_over_one_long_sequence(n, d, store):
    """From one workgroup to a thousand splits; sharp weights, the largest in the last position."""
    page = 64
    cache = fx.KVCache.empty(-(-n // page), page, 1, d, torch.float8_e4m3fn if store == "e4m3" else torch.bfloat16)
    table = torch.from_numpy(np.random.default_rng(n).permutation(-(-n // page)).astype(np.int32)).cuda()[None]
    k, k64 = draw(1, n, 1, d, "bf16")
    v, v64 = draw(2, n, 1, d, "bf16")
    q, q64 = draw(3, 1, 3, d, "bf16", std=3.0)
    k[-1, 0] = q[0, 1]
    k64[-1, 0] = q64[0, 1]
    fx.cache_write(cache, table, torch.zeros(1, dtype=torch.int32, device="cuda"), k, v, seqs=fx.build_sequences([[0, n]]))
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    out, lse = fx.attention_step(cache, table, lens, q)
    ro, rl, bo, bl = A.attention(q64, _held(k64, store), _held(v64, store), [0, 1], [0, n], False, d ** -0.5, "bf16")
    A.check(_f64(out), ro, bo, "bf16", "out")
    A.check(_f64(lse), rl.T, bl.T, "f32", "lse")
    again = fx.attention_step(cache, table, lens, q)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


def test_pages_that_sequences_share():
    """A prompt's pages in the tables of four sequences, each with a last page of its own."""
    page, d = 16, 32
    cache = fx.KVCache.empty(20, page, 2, d, torch.float16)
    k, k64 = draw(1, 64, 2, d, "f16")
    v, v64 = draw(2, 64, 2, d, "f16")
    table = torch.tensor([[5, 9, 2, 10 + i] for i in range(4)], dtype=torch.int32, device="cuda")
    fx.cache_write(cache, table[:1], torch.zeros(1, dtype=torch.int32, device="cuda"), k[:48], v[:48], seqs=fx.build_sequences([[0, 48]]))
    at = torch.full((4,), 48, dtype=torch.int32, device="cuda")
    fx.cache_write(cache, table, at, k[48:52], v[48:52])
    q, q64 = draw(3, 4, 4, d, "f16")
    out, _ = fx.attention_step(cache, table, at + 1, q)
    each = [np.concatenate([np.concatenate([x[:48], x[48 + i:49 + i]]) for i in range(4)]) for x in (k64, v64)]
    ro, _, bo, _ = A.attention(q64, *each, np.arange(5), 49 * np.arange(5), False, d ** -0.5, "f16")
    A.check(_f64(out), ro, bo, "f16", "out")


def test_infinities_behind_a_length():
    """What lies in a page behind a sequence's length, and in pages of others, is not looked at, NaN too."""
    page, d = 16, 64
    for dtype in (torch.bfloat16, torch.float32):
        cache = fx.KVCache.empty(6, page, 1, d, dtype)
        cache.k.fill_(float("nan"))
        cache.v.fill_(float("inf"))
        k, v = (torch.randn((21, 1, d), device="cuda").to(dtype) for _ in range(2))
        table, zero = torch.tensor([[4, 1, 2]], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        fx.cache_write(cache, table, zero, k, v, seqs=fx.build_sequences([[0, 21]]))
        q = torch.randn((1, 2, d), device="cuda").to(dtype)
        out, lse = fx.attention_step(cache, table, zero + 21, q)
        ref, rl, bo, bl = A.attention(_f64(q), _f64(k), _f64(v), [0, 1], [0, 21], False, d ** -0.5, "f32" if dtype == torch.float32 else "bf16")
        A.check(_f64(out), ref, bo, "f32" if dtype == torch.float32 else "bf16", "out")
        A.check(_f64(lse), rl.T, bl.T, "f32", "lse")


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("kv_lens", [None, [70, 9]])
def test_gradients_are_the_differences(causal, kv_lens):
    """Of a weighted sum of both outputs in fp32, along one direction for each input, by 2^-6 either side: third derivatives stay
    below a per cent of the directional derivative's scale |gradient| |direction|."""
    lens, heads, kvh, d = [40, 61], 4, 2, 24
    seqs = fx.build_sequences(_joff(lens)[1])
    kv = None if kv_lens is None else fx.build_sequences(_joff(kv_lens)[1])
    n, m = sum(lens), sum(kv_lens or lens)
    gen = torch.Generator(device="cuda").manual_seed(5)
    new = lambda *s: torch.randn(s, generator=gen, device="cuda")
    t = [new(n, heads, d), new(m, kvh, d), new(m, kvh, d)]
    go, gl = new(n, heads, d), new(heads, n)

    def value(t):
        out, lse = fx.attention_fwd(seqs, *t, causal=causal, kv_seqs=kv)
        return float((out.double() * go).sum() + torch.where(torch.isfinite(lse), lse.double() * gl, 0.0).sum())
    out, lse = fx.attention_fwd(seqs, *t, causal=causal, kv_seqs=kv)
    grads = fx.attention_bwd(seqs, *t, out, lse, go, grad_lse=gl, causal=causal, kv_seqs=kv)
    for i, g in enumerate(grads):
        direction = new(*g.shape)
        direction /= direction.norm()
        e = 2.0 ** -6
        up, down = ([x + s * e * direction if j == i else x for j, x in enumerate(t)] for s in (1, -1))
        assert abs((value(up) - value(down)) / (2 * e) - float((g * direction).sum())) <= 1e-2 * float(g.norm()) + 1e-6


def test_gradients_that_are_not_asked_for():
    lens, heads, kvh, d = [90, 0, 40], 4, 2, 64
    b, jo = _joff(lens)
    n = int(b[-1])
    seqs = fx.build_sequences(jo)
    q, k, v, go = (draw(i, n, h, d, "bf16")[0] for i, h in enumerate((heads, kvh, kvh, heads)))
    out, lse = fx.attention_fwd(seqs, q, k, v)
    ref = fx.attention_bwd(seqs, q, k, v, out, lse, go)
    a = B._attention(seqs, None, q, k, v, False, None, torch.cuda.current_device())
    for which in range(8):
        got = [torch.full_like(r, 3.0) for r in ref]
        outs = [x for i, (t, h) in enumerate(zip(got, (heads, kvh, kvh))) for x in ((t.data_ptr() if which >> i & 1 else None), h * d, d)]
        assert B.lib.fx_attention_bwd(C.byref(a), out.data_ptr(), heads * d, d, lse.data_ptr(), go.data_ptr(), heads * d, d, None, *outs, B._stream()) == 0
        torch.cuda.synchronize()
        for i, (x, r) in enumerate(zip(got, ref)):
            assert torch.equal(x, r) if which >> i & 1 else (x == 3.0).all()
    assert B.lib.fx_attention_fwd(C.byref(a), out.data_ptr(), heads * d, d, None, B._stream()) == 0


@pytest.mark.parametrize("causal", [False, True])
def test_many_short_sequences(causal):
    rng = np.random.default_rng(1)
    run(list(rng.integers(0, 5, 4000)), 2, 1, 16, "f16", causal)
    run(list(rng.integers(0, 40, 600)), 3, 3, 32, "bf16", causal, layout="columns")


# rows, heads and widths of every way to share them out: blocks of 32 with eight or four waves, two blocks that share tiles, tiles of 64 and 128
@pytest.mark.parametrize("lens,heads,kv_heads,d,dtype", [
    ([700], 2, 1, 64, "bf16"), ([700], 2, 1, 128, "f16"), ([600], 1, 1, 256, "bf16"), ([500], 2, 2, 64, "f32"), ([300], 1, 1, 200, "f32"),
    ([900, 800], 8, 8, 64, "bf16"), ([900, 800], 8, 8, 64, "f32"), ([700, 900], 8, 8, 128, "bf16"), ([500, 700], 8, 8, 256, "f16"), ([300, 500], 12, 12, 140, "f32"),
    ([100] * 20 + [40] * 30, 16, 8, 32, "bf16"), ([1200, 1000], 16, 16, 64, "f16"), ([700, 900], 24, 12, 128, "bf16"), ([900, 700], 24, 24, 40, "f32")])
@pytest.mark.parametrize("causal", [False, True])
def test_ways_to_share_out(lens, heads, kv_heads, d, dtype, causal):
    run(lens, heads, kv_heads, d, dtype, causal)


def test_sequences_by_size():
    """Long, short and empty ones in any order, more heads than eight and not a multiple; keys of another set, some longer, some none."""
    lens = [5, 2300, 0, 64, 1, 700, 33, 2, 0, 129]
    run(lens, 3, 1, 32, "bf16", True, kv_lens=[900, 40, 7, 0, 300, 700, 1, 2, 0, 2000])
    run(lens, 8, 8, 32, "f16", True)
    run(lens, 8, 4, 64, "bf16", False)


@pytest.mark.parametrize("dtype,d", [("f16", 200), ("f32", 140), ("bf16", 33)])
def test_wide_rows_do_not_see_what_comes_later(dtype, d):
    """One value of the last row of a causal sequence not finite, in each input: the rows and keys that do not see it against the formulas."""
    n, heads, kvh = 75, 2, 1
    seqs = fx.build_sequences([[0, n]])
    make = lambda: [draw(s, n, h, d, dtype)[0] for s, h in ((1, heads), (2, kvh), (3, kvh), (4, heads))]
    t = make()
    f = [_f64(x) for x in t]
    out, lse = fx.attention_fwd(seqs, *t[:3], causal=True)
    ro, _, bo, _ = A.attention(*f[:3], [0, n], [0, n], True, d ** -0.5, dtype)
    rg = A.attention_grad(*f, [0, n], [0, n], True, d ** -0.5, dtype)
    for which in range(4):
        for c in (0, d - 1):
            u = make()
            u[which][n - 1, 0, c] = float("nan")
            o, _ = fx.attention_fwd(seqs, *u[:3], causal=True)
            A.check(_f64(o)[:-1], ro[:-1], bo[:-1], dtype, f"out, {which}")
            g = fx.attention_bwd(seqs, *u[:3], out, lse, u[3], causal=True)
            if which in (1, 2):
                A.check(_f64(g[0])[:-1], rg[0][:-1], rg[3][:-1], dtype, f"gq, {which}")
            else:               # a row in the middle of a block: keys behind it do not see it
                u = make()
                u[which][40, 0, c] = float("inf")
                g = fx.attention_bwd(seqs, *u[:3], out, lse, u[3], causal=True)
                for i in (1, 2):
                    A.check(_f64(g[i])[41:], rg[i][41:], rg[3 + i][41:], dtype, f"gradient {i}, {which}")


def test_nothing_finite():
    """A causal pass over NaN alone ends in about the time of any other, and is NaN; so is one with a channel of NaN, in that channel."""
    n, heads, d = 16_384, 8, 64
    seqs = fx.build_sequences([[0, n]])
    x = torch.full((n, heads, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    out, lse = fx.attention_fwd(seqs, x, x, x, causal=True)
    g = fx.attention_bwd(seqs, x, x, x, out, lse, x, causal=True)
    assert all(torch.isnan(t).all() for t in (out, lse, *g))
    q, k, v, go = (draw(s, n, heads, d, "bf16")[0] for s in range(4))
    ref, _ = fx.attention_fwd(seqs, q, k, v, causal=True)
    v[:, :, 5] = float("nan")
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    out, lse = fx.attention_fwd(seqs, q, k, v, causal=True)
    end.record()
    torch.cuda.synchronize()
    assert start.elapsed_time(end) < 500
    clean = [c for c in range(d) if c != 5]
    assert torch.isnan(out[:, :, 5]).all() and torch.equal(out[:, :, clean], ref[:, :, clean])
    go[:, :, 7] = float("inf")
    g = fx.attention_bwd(seqs, q, k, v, out, lse, go, causal=True)
    assert not torch.isfinite(g[2][:, :, 7]).any() and torch.isfinite(g[2][:, :, clean[:5]]).all()


def test_no_queries():
    kv = fx.build_sequences([[0, 5], [5, 5]])
    none = fx.build_sequences([[0, 0], [0, 0]])
    q, k = torch.zeros((0, 4, 32), device="cuda"), torch.randn((5, 2, 32), device="cuda")
    out, lse = fx.attention_fwd(none, q, k, k, kv_seqs=kv)
    g = fx.attention_bwd(none, q, k, k, out, lse, q, kv_seqs=kv)
    assert out.shape == (0, 4, 32) and lse.shape == (4, 0) and g[0].shape == q.shape and not g[1].any() and not g[2].any()


@pytest.mark.parametrize("n,heads,kv_heads,dim,dtype,store", [(300, 3, 1, 64, "bf16", "bf16"), (70, 8, 4, 40, "f32", "f32"), (260, 4, 2, 128, "f16", "e4m3")])
def test_step_of_more_sequences_than_compute_units(n, heads, kv_heads, dim, dtype, store):
    """One workgroup of four waves for each, several on a unit."""
    rng = np.random.default_rng(n)
    lens = rng.integers(0, 200, size=n).tolist()
    lens[0], lens[-1] = 0, 1
    bounds, jo = _joff(lens)
    table, pages = _tables(rng, lens, 16)
    cache = fx.KVCache.empty(pages, 16, kv_heads, dim, torch.float8_e4m3fn if store == "e4m3" else {"bf16": torch.bfloat16, "f32": torch.float32}[store])
    k, k64 = draw(1, bounds[-1], kv_heads, dim, dtype)
    v, v64 = draw(2, bounds[-1], kv_heads, dim, dtype)
    q, q64 = draw(3, n, heads, dim, dtype, std=2.0)
    fx.cache_write(cache, table, torch.zeros(n, dtype=torch.int32, device="cuda"), k, v, seqs=fx.build_sequences(jo))
    out, lse = fx.attention_step(cache, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), q)
    ro, rl, bo, bl = A.attention(q64, _held(k64, store), _held(v64, store), np.arange(n + 1), bounds, False, dim ** -0.5, dtype)
    A.check(_f64(out), ro, bo, dtype, "out")
    A.check(_f64(lse), rl.T, bl.T, "f32", "lse")


@pytest.mark.parametrize("lens,d,dtype", [([4200] + [300] * 100, 128, "f16"), ([4200] + [300] * 100, 40, "f32"), ([4096] * 8, 200, "bf16")])
def test_keys_whose_queries_two_workgroups_share(lens, d, dtype):
    run(lens, 1, 1, d, dtype, True)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f16", 128)])
def test_shared_queries_that_are_not_finite(dtype, d):
    """A query and its gradient of NaN in one channel: keys behind them do not see it, whichever workgroup had them."""
    n, at = 4200, 2000
    seqs = fx.build_sequences(_joff([n] + [300] * 100)[1])
    t = [draw(s, seqs.rows, 1, d, dtype)[0] for s in (1, 2, 3, 4)]
    rg = A.attention_grad(*[_f64(x)[:n] for x in t], [0, n], [0, n], True, d ** -0.5, dtype)
    out, lse = fx.attention_fwd(seqs, *t[:3], causal=True)
    t[0][at, 0, 1] = t[3][at, 0, d - 1] = float("nan")
    g = fx.attention_bwd(seqs, *t[:3], out, lse, t[3], causal=True)
    for i in (1, 2):
        A.check(_f64(g[i])[at + 1:n], rg[i][at + 1:], rg[3 + i][at + 1:], dtype, f"gradient {i}")
        assert torch.isnan(g[i][:at + 1]).any() and torch.isfinite(g[i][n:]).all()
