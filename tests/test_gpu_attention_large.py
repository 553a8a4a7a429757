"""Offsets that pass 32 bits: rows of attention and of a cache behind the fourth GiB of their tensors; and rows beyond a result,
left as they were."""
import numpy as np
import pytest
import torch

import attention_reference as A
import paper_2407_01781_amd as fx

pytestmark = pytest.mark.gpu


def _f64(t):
    return t.double().cpu().numpy()


def test_rows_behind_four_gib():
    """Heads that are columns of rows of 64 KiB, 70,000 rows; the last two sequences against the formulas."""
    n, wide, d = 70_000, 512, 64
    lens = [69_000, 300, 0, 700]
    b = np.concatenate([[0], np.cumsum(lens)])
    base = torch.zeros((n, wide, d), dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    for s in (slice(500, 502), slice(504, 505), slice(508, 509)):
        base[:, s] = torch.randn((n, s.stop - s.start, d), generator=gen, device="cuda").bfloat16()
    q, k, v = base[:, 500:502], base[:, 504:505], base[:, 508:509]
    seqs = fx.build_sequences(np.stack([b[:-1], b[1:]], 1))
    out = base[:, 400:402]                  # the result lies in the same rows
    _, lse = fx.attention_fwd(seqs, q, k, v, causal=True, out=out)
    go = torch.randn((n, 2, d), generator=gen, device="cuda").bfloat16()
    g = fx.attention_bwd(seqs, q, k, v, out, lse, go, causal=True)
    at = slice(69_000, 70_000)
    local = np.array([0, 300, 300, 1000])
    t = [_f64(x[at]) for x in (q, k, v, go)]
    ro, rl, bo, bl = A.attention(*t[:3], local, local, True, d ** -0.5, "bf16")
    A.check(_f64(out[at]), ro, bo, "bf16", "out")
    A.check(_f64(lse[:, at]), rl, bl, "f32", "lse")
    rg = A.attention_grad(*t, local, local, True, d ** -0.5, "bf16")
    for x, y, e in zip(g, rg[:3], rg[3:]):
        A.check(_f64(x[at]), y, e, "bf16", "gradient")
    assert not base[:, 402:500].any() and not base[:, :400].any()


@pytest.mark.parametrize("store", ["f32", "e4m3"])
def test_pages_behind_four_gib(store):
    d, page, kvh = 256, 256, 1
    per = page * d * (4 if store == "f32" else 1)
    pages = (5 << 30) // per
    cache = fx.KVCache.empty(pages, page, kvh, d, torch.float32 if store == "f32" else torch.float8_e4m3fn)
    lens = [600, 1300, 40]
    b = np.concatenate([[0], np.cumsum(lens)])
    gen = torch.Generator(device="cuda").manual_seed(2)
    k, v = (torch.randn((b[-1], kvh, d), generator=gen, device="cuda") for _ in range(2))
    table = np.full((3, 6), -1, np.int32)
    table[0, :3], table[1], table[2, 0] = [pages - 1, 0, pages - 5], pages - 10 - np.arange(6), pages - 2
    table = torch.from_numpy(table).cuda()
    zero, seqs = torch.zeros(3, dtype=torch.int32, device="cuda"), fx.build_sequences(np.stack([b[:-1], b[1:]], 1))
    fx.cache_write(cache, table, zero, k, v, seqs=seqs)
    rk, rv = fx.cache_read(cache, table, zero, seqs, dtype=torch.float32)
    held = [_f64(k), _f64(v)] if store == "f32" else [A.quantised(_f64(k)), A.quantised(_f64(v))]
    assert np.array_equal(_f64(rk), held[0]) and np.array_equal(_f64(rv), held[1])
    q = torch.randn((3, 3, d), generator=gen, device="cuda")
    out, lse = fx.attention_step(cache, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), q)
    ro, rl, bo, bl = A.attention(_f64(q), *held, np.arange(4), b, False, d ** -0.5, "f32")
    A.check(_f64(out), ro, bo, "f32", "out")
    A.check(_f64(lse), rl.T, bl.T, "f32", "lse")


def test_what_lies_around_results_stays():
    """Results that are column ranges of wider rows, of every kind of row: nothing else of those is written."""
    lens, kvh, heads = [70, 33], 2, 4
    seqs = fx.build_sequences([[0, 70], [70, 103]])
    for dtype, d in ((torch.bfloat16, 64), (torch.float16, 37), (torch.float32, 12)):
        gen = torch.Generator(device="cuda").manual_seed(3)
        q, k, v = (torch.randn((sum(lens), h, d), generator=gen, device="cuda").to(dtype) for h in (heads, kvh, kvh))
        wide = torch.full((sum(lens) + 2, heads + 2, d + 8), 5.0, dtype=dtype, device="cuda")
        out = wide[1:-1, 1:-1, 4:-4]
        assert torch.equal(fx.attention_fwd(seqs, q, k, v, out=out)[0], fx.attention_fwd(seqs, q, k, v)[0])
        keep = torch.ones_like(wide, dtype=torch.bool)
        keep[1:-1, 1:-1, 4:-4] = False
        assert (wide[keep] == 5.0).all()
        cache = fx.KVCache.empty(8, 16, kvh, d, dtype)
        table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
        fx.cache_write(cache, table, torch.zeros(2, dtype=torch.int32, device="cuda"), k[:100], v[:100], seqs=fx.build_sequences([[0, 60], [60, 100]]))
        wide.fill_(5.0)
        lens_on = torch.tensor([60, 40], dtype=torch.int32, device="cuda")
        small = wide[1:3, 1:-1, 4:-4]
        ref = fx.attention_step(cache, table, lens_on, q[:2])[0]
        assert torch.equal(fx.attention_step(cache, table, lens_on, q[:2], out=small)[0], ref)
        keep[3:-1] = True
        assert (wide[keep] == 5.0).all()
