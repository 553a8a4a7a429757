"""One value that is not finite near the end of a long causal sequence: the passes end in about the time of any other, and rows and
keys that do not see it are what they are without it."""
import numpy as np
import pytest
import torch

import attention_reference as A
import paper_2407_01781_amd as fx
from test_gpu_attention import _f64, _joff, draw

pytestmark = pytest.mark.gpu


def _ms(run):
    """The shortest of three."""
    best = float("inf")
    for _ in range(3):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        out = run()
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b))
    return best, out


@pytest.mark.parametrize("heads,kv_heads,d,dtype,bad", [(4, 2, 64, "f16", float("inf")), (4, 1, 128, "bf16", float("nan")), (2, 2, 64, "f32", float("-inf"))])
@pytest.mark.parametrize("which", ["v", "k", "q", "gout"])
def test_time(heads, kv_heads, d, dtype, bad, which):
    """Two of 16,384 rows, one in the last tile and one in the middle, whose blocks every later row passes: up to twice the time and half a
    millisecond (a wave then goes over at most a few hundred rows again, at some microseconds each)."""
    n = 16_384
    seqs = fx.build_sequences([[0, n]])
    t = {name: draw(s, n, h, d, dtype)[0] for s, (name, h) in enumerate((("q", heads), ("k", kv_heads), ("v", kv_heads), ("gout", heads)))}
    fwd = lambda: fx.attention_fwd(seqs, t["q"], t["k"], t["v"], causal=True)
    clean, (out, lse) = _ms(fwd)
    bwd = lambda: fx.attention_bwd(seqs, t["q"], t["k"], t["v"], out, lse, t["gout"], causal=True)
    clean_bwd, grads = _ms(bwd)
    rows = (n - 9, n // 2 + 5)
    for r in rows:
        t[which][r, -1, 3] = bad
    ms, (odd, _) = _ms(fwd)
    ms_bwd, odd_grads = _ms(bwd)
    print(f"{which}: {clean:.2f} -> {ms:.2f} ms, gradients {clean_bwd:.2f} -> {ms_bwd:.2f}")
    assert torch.equal(odd[:rows[1]], out[:rows[1]])
    if which in "vk":
        assert torch.equal(odd_grads[0][:rows[1]], grads[0][:rows[1]])
    else:
        assert all(torch.equal(odd_grads[i][rows[0] + 1:], grads[i][rows[0] + 1:]) for i in (1, 2))
    assert ms <= 2 * clean + 0.5 and ms_bwd <= 2 * clean_bwd + 0.5


@pytest.mark.parametrize("lens,kv_lens,heads,kv_heads,d,dtype", [
    ([700], None, 2, 1, 64, "bf16"), ([500, 300], None, 4, 2, 128, "f16"), ([300], [420], 3, 1, 40, "f32"), ([150] * 30, None, 4, 4, 32, "bf16"),
    ([2000, 90], None, 16, 8, 64, "f16"), ([900], None, 8, 8, 128, "bf16"), ([70], [33], 2, 2, 200, "bf16"), ([330], None, 2, 2, 200, "f32"), ([4300] + [300] * 100, None, 1, 1, 64, "bf16"),
    ([12, 60, 33, 9], None, 4, 2, 64, "f16"), ([1, 2, 5, 16, 17, 3], None, 3, 1, 32, "bf16"), ([16, 4], [7, 30], 2, 2, 128, "bf16"), ([15], None, 1, 1, 200, "f16")])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_seen_and_unseen(lens, kv_lens, heads, kv_heads, d, dtype, bad):
    """Every element of out and gv against the formula where a value, or an output's gradient, is not finite: what does not see it is
    finite, what does see it is not, and of the same kind.  Of the rest the rows and keys that do not see it."""
    bq, jq = _joff(lens)
    bk, jk = (bq, jq) if kv_lens is None else _joff(kv_lens)
    seqs, kv = fx.build_sequences(jq), None if kv_lens is None else fx.build_sequences(jk)
    make = lambda: [draw(s, m[-1], h, d, dtype)[0] for s, m, h in ((1, bq, heads), (2, bk, kv_heads), (3, bk, kv_heads), (4, bq, heads))]
    t = make()
    f = [_f64(x) for x in t]
    ro, _, bo, _ = A.attention(*f[:3], bq, bk, True, d ** -0.5, dtype)
    rg = A.attention_grad(*f, bq, bk, True, d ** -0.5, dtype)
    out, lse = fx.attention_fwd(seqs, *t[:3], causal=True, kv_seqs=kv)
    rng = np.random.default_rng(3)
    g = heads // kv_heads
    for which in range(4):
        u = make()
        b = (bq, bk, bk, bq)[which]
        head, c = u[which].shape[1] - 1, int(rng.integers(d))
        rows = [int(rng.integers(max(b[s], b[s + 1] - 70), b[s + 1])) for s in range(len(b) - 1)]
        for r in rows:
            u[which][r, head, c] = bad
        o, _ = fx.attention_fwd(seqs, *u[:3], causal=True, kv_seqs=kv)
        got = [_f64(x) for x in fx.attention_bwd(seqs, *u[:3], out, lse, u[3], causal=True, kv_seqs=kv)]
        heads_of = slice(head * g, head * g + g)
        for s, r in enumerate(rows):
            q0, q1, k0, k1 = bq[s], bq[s + 1], bk[s], bk[s + 1]
            if which in (1, 2):
                first = max(q0, q1 - (k1 - r))              # the first query that sees the key
                A.check(_f64(o)[q0:first], ro[q0:first], bo[q0:first], dtype, "out")
                A.check(got[0][q0:first], rg[0][q0:first], rg[3][q0:first], dtype, "gq")
                if which == 2:
                    want = ro[first:q1].copy()
                    want[:, heads_of, c] = bad
                    A.check(_f64(o)[first:q1], want, bo[first:q1], dtype, "out of rows that see it")
                else:
                    assert not np.isfinite(got[0][first:q1, heads_of, c]).any()
            else:
                last = min(k1, k1 - (q1 - r) + 1)           # keys from here on are not seen by the row
                last = max(last, k0)
                for i in (1, 2):
                    A.check(got[i][last:k1], rg[i][last:k1], rg[3 + i][last:k1], dtype, f"gradient {i}")
                if which == 3:
                    want = rg[2][k0:last].copy()
                    want[:, head // g, c] = bad
                    A.check(got[2][k0:last], want, rg[5][k0:last], dtype, "gv of keys that see it")


def _seen(dtype, d, n, bad):
    """Two queries over n keys each, values of which some are not finite, what comes of them and its bound."""
    heads, kvh, seqs = 4, 2, 2
    b, jo = _joff([n] * seqs)
    (q, q64), (k, k64), (v, v64) = (draw(s, m, h, d, dtype) for s, m, h in ((1, seqs, heads), (2, n * seqs, kvh), (3, n * seqs, kvh)))
    ro, _, bo, _ = A.attention(q64, k64, v64, np.arange(seqs + 1), b, False, d ** -0.5, dtype)
    at = np.random.default_rng(n).integers(n, size=4)
    want = ro.copy()
    for i, c in enumerate((1, d - 1)):
        v[at[i], 1, c] = bad
        want[0, 2:, c] = bad
    if n > 1:
        v[n + (at[2] + 1) % n, 0, 2], v[n + at[2], 0, 2] = float("inf"), float("-inf")
        want[1, :2, 2] = np.nan
    return q, k, v, fx.build_sequences(jo), want, bo


SEEN = [pytest.mark.parametrize("dtype,d", [("f16", 64), ("bf16", 40), ("f32", 64), ("bf16", 200), ("f16", 128)]),
        pytest.mark.parametrize("n", [1, 2, 16, 17, 33, 700, 5000]), pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])]


@SEEN[0]
@SEEN[1]
@SEEN[2]
def test_values_that_a_step_sees(dtype, d, n, bad):
    """An infinity in a value is what every row that sees it has there; two that differ in sign, or a NaN, are a NaN; the other channels are as without."""
    q, k, v, keys, want, bound = _seen(dtype, d, n, bad)
    cache = fx.KVCache.empty(2 * -(-n // 16), 16, 2, d, k.dtype)
    table = torch.randperm(cache.k.shape[0], generator=torch.Generator().manual_seed(1)).to(torch.int32).view(2, -1).cuda()
    fx.cache_write(cache, table, torch.zeros(2, dtype=torch.int32, device="cuda"), k, v, seqs=keys)
    out, _ = fx.attention_step(cache, table, torch.full((2,), n, dtype=torch.int32, device="cuda"), q)
    A.check(_f64(out), want, bound, dtype, "step")


@SEEN[0]
@SEEN[1]
@SEEN[2]
def test_values_that_rows_see(dtype, d, n, bad):
    q, k, v, keys, want, bound = _seen(dtype, d, n, bad)
    A.check(_f64(fx.attention_fwd(fx.build_sequences([[0, 1], [1, 2]]), q, k, v, kv_seqs=keys)[0]), want, bound, dtype, "forward")


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("lens", [[1, 2, 8, 16, 30], [1, 2, 9, 16, 40, 200]])
def test_gradients_of_few_rows(dtype, bad, lens):
    """An infinity in an output's gradient is what the values that its row sees have there, over few rows and many."""
    heads, kvh, d = 2, 1, 64
    b, jo = _joff(lens)
    seqs = fx.build_sequences(jo)
    t = [draw(s, b[-1], h, d, dtype)[0] for s, h in ((1, heads), (2, kvh), (3, kvh), (4, heads))]
    ref = A.attention_grad(*[_f64(x) for x in t], b, b, False, d ** -0.5, dtype)
    out, lse = fx.attention_fwd(seqs, *t[:3])
    want = ref[2].copy()
    for s in range(len(lens)):
        t[3][int(b[s]) + lens[s] // 2, 1, 5] = bad
        want[b[s]:b[s + 1], 0, 5] = bad
    _, _, gv = fx.attention_bwd(seqs, *t[:3], out, lse, t[3])
    A.check(_f64(gv), want, ref[5], dtype, "gv")
