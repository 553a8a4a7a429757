"""Attention in fp16 where weights and gradients of scores are small: fp16's least number is 2^-24, a weight is about 1 / keys, and an
output may be far above both.  The bounds are those of attention_reference.py with the least number that the kernels'
powers of two leave in the place of the type's."""
from unittest import mock

import numpy as np
import pytest
import torch

import attention_reference as A
import paper_2407_01781_amd as fx
from test_gpu_attention import _f64, _joff, draw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,heads,kv_heads,d", [([4096], 2, 1, 64), ([300, 0, 2500], 4, 2, 32), ([1030] * 3, 1, 1, 128), ([700, 90], 2, 2, 200),
                                                   ([120] * 40, 4, 4, 32), ([4200] + [300] * 100, 1, 1, 64)])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("std", [1e-3, 1e-5])
def test_small_gradients_of_the_output(lens, heads, kv_heads, d, causal, std):
    """Gradients are linear in the output's, and so are their bounds, but for fp16's least number: with gout times 2^20 it is 2^-20 of
    itself beside them.  Keys of 2^-6 and a scale of 2^12 leave the scores and make the gradients large enough for fp16."""
    b, jo = _joff(lens)
    seqs, scale, up = fx.build_sequences(jo), 2.0 ** 12 * d ** -0.5, 2.0 ** 20
    (q, q64), (k, k64) = (draw(s, b[-1], h, d, "f16", std=2.0 ** -6) for s, h in ((1, heads), (2, kv_heads)))
    v, v64 = draw(3, b[-1], kv_heads, d, "f16")
    go, go64 = draw(4, b[-1], heads, d, "f16", std=std)
    out, lse = fx.attention_fwd(seqs, q, k, v, causal=causal, scale=scale)
    got = fx.attention_bwd(seqs, q, k, v, out, lse, go, causal=causal, scale=scale)
    ref = [x / up for x in A.attention_grad(q64, k64, v64, go64 * up, b, b, causal, scale, "f16")]
    for name, x, y, e in list(zip(("gq", "gk", "gv"), got, ref[:3], ref[3:])):
        if name != "gv":            # there it is the weight's own, below
            A.check(_f64(x), y, e, "f16", name)


@pytest.mark.parametrize("queries,keys,heads,kv_heads,d,causal", [([64], [262_144], 1, 1, 64, False), ([40, 3], [90_000, 150_000], 2, 1, 32, True), ([130], [70_000], 2, 2, 128, True)])
def test_small_weights_of_the_gradients(queries, keys, heads, kv_heads, d, causal):
    """Weights of some 2^-18: what the kernels lose of one is 2^-40 at most, and of a gradient of a score 2^-32 of its row's largest, here 2^-10."""
    bq, jq = _joff(queries)
    bk, jk = _joff(keys)
    seqs, kv = fx.build_sequences(jq), fx.build_sequences(jk)
    q, q64 = draw(1, bq[-1], heads, d, "f16")
    (k, k64), (v, v64) = (draw(s, bk[-1], kv_heads, d, "f16") for s in (2, 3))
    go, go64 = draw(4, bq[-1], heads, d, "f16", std=50.0)
    out, lse = fx.attention_fwd(seqs, q, k, v, causal=causal, kv_seqs=kv)
    got = fx.attention_bwd(seqs, q, k, v, out, lse, go, causal=causal, kv_seqs=kv)
    with mock.patch.dict(A.LEAST, f16=2.0 ** -40):
        ref = A.attention_grad(q64, k64, v64, go64, bq, bk, causal, d ** -0.5, "f16")
    for name, x, y, e in zip(("gq", "gk", "gv"), got, ref[:3], ref[3:]):
        A.check(_f64(x), y, e, "f16", name)


def _one_leads(n, heads, d, nats, dtype, rows=1):
    """Queries and keys of which key 5 leads the others by so many nats, all in a channel of their own; values of about 1, its own 0."""
    q, _ = draw(1, rows, heads, d, dtype, std=0.02)
    k, _ = draw(2, n, 1, d, dtype, std=0.02)
    v, _ = draw(3, n, 1, d, dtype, std=0.1)
    q[..., 0], k[..., 0], k[5, :, 0] = d ** 0.5, 0.0, nats
    v += 1
    v[5] = 0
    return q, k, v


@pytest.mark.parametrize("n,nats,heads,d,rows", [(100_000, 15.0, 1, 64, 40), (100_000, 17.0, 2, 32, 200), (60_000, 19.0, 1, 128, 300), (3_000, 16.0, 4, 64, 2_000), (60, 14.0, 2, 64, 3)])
def test_one_key_leads(n, nats, heads, d, rows):
    """What a weight loses below fp16's normal numbers is 2^-36 of the row's largest at most, however many keys there are."""
    q, k, v = _one_leads(n, heads, d, nats, "f16", rows)
    f = [_f64(x) for x in (q, k, v)]
    seqs, kv = fx.build_sequences([[0, rows]]), fx.build_sequences([[0, n]])
    out, lse = fx.attention_fwd(seqs, q, k, v, kv_seqs=kv)
    with mock.patch.dict(A.LEAST, f16=2.0 ** -36 / 256):            # the bound takes 256 of it, of the row's largest
        ro, rl, bo, bl = A.attention(*f, [0, rows], [0, n], False, d ** -0.5, "f16")
    A.check(_f64(lse), rl, bl, "f32", "lse")
    A.check(_f64(out), ro, bo, "f16", "out")


def _cached(k, v, dtype, store=None, page=256):
    """Rows of one sequence in a cache, and its table."""
    n, kvh, d = k.shape
    pages = -(-n // page)
    cache = fx.KVCache.empty(pages, page, kvh, d, store or k.dtype)
    table = torch.arange(pages, dtype=torch.int32, device="cuda").flip(0)[None].contiguous()
    fx.cache_write(cache, table, torch.zeros(1, dtype=torch.int32, device="cuda"), k, v, seqs=fx.build_sequences([[0, n]]))
    return cache, table


# half units of what a step's weights keep where they meet values: two parts of the cache's type, three of bf16 with fp32 queries over 8 bits
STEP = {("bf16", None): 2.0 ** -16, ("f16", None): 2.0 ** -22, ("f32", None): 2.0 ** -24, ("bf16", "e4m3"): 2.0 ** -16, ("f16", "e4m3"): 2.0 ** -16, ("f32", "e4m3"): 2.0 ** -24}


def _step_bounds(q, k, v, bounds, dtype, store):
    """Of one row over all keys of its sequence: weights as the step has them; where they are fp16 they lose 2^-40 of the largest beside that."""
    with mock.patch.dict(A.HALF, step=STEP[dtype, store]), mock.patch.dict(A.LEAST, step=2.0 ** -40 / 256 if dtype == "f16" and not store else 0.0):
        return A.attention(q, k, v, np.arange(len(bounds)), bounds, False, q.shape[2] ** -0.5, "step")


@pytest.mark.parametrize("n,nats,heads,d,dtype", [(986_880, 15.0, 1, 64, "f16"), (986_880, 17.0, 2, 16, "f16"), (100_000, 20.0, 1, 64, "f16"), (900, 15.0, 8, 128, "f16"), (100_000, 20.0, 1, 64, "bf16"), (5_000, 17.0, 2, 200, "f16")])
def test_one_key_leads_a_step(n, nats, heads, d, dtype):
    q, k, v = _one_leads(n, heads, d, nats, dtype)
    cache, table = _cached(k, v, dtype)
    out, lse = fx.attention_step(cache, table, torch.tensor([n], dtype=torch.int32, device="cuda"), q)
    ro, rl, bo, bl = _step_bounds(_f64(q), _f64(k), _f64(v), [0, n], dtype, None)
    A.check(_f64(lse), rl.T, bl.T, "f32", "lse")
    A.check(_f64(out), ro, bo, dtype, "out")


@pytest.mark.parametrize("dtype,store", list(STEP))
@pytest.mark.parametrize("n,heads,d", [(2, 1, 64), (7, 2, 64), (40, 3, 128), (300, 1, 33), (3000, 2, 256), (9, 16, 16)])
def test_digits_of_a_step(n, heads, d, dtype, store):
    """Values that nearly cancel show what the weights are rounded to: in one part it would be 2^-9 or 2^-12 of the sum's size."""
    seqs = 5
    bounds, jo = _joff([n] * seqs)
    (q, q64), (k, k64), (v, v64) = (draw(s, m, h, d, dtype) for s, m, h in ((1, seqs, heads), (2, n * seqs, 1), (3, n * seqs, 1)))
    to = torch.float8_e4m3fn if store else v.dtype
    held = lambda x: A.quantised(x) if store else x
    for i in range(seqs):               # the last value of each sequence cancels the others under the first head's weights
        part = slice(i * n, i * n + n)
        p = np.exp(d ** -0.5 * (held(k64[part, 0]) @ q64[i, 0]))
        v64[i * n + n - 1, 0] = -(p[:-1] @ held(v64[part, 0])[:-1]) / p[-1]
    v = torch.from_numpy(v64).to(v.dtype).cuda()
    v64 = _f64(v)
    page = 16
    cache = fx.KVCache.empty(seqs * -(-n // page), page, 1, d, to)
    table = torch.randperm(cache.k.shape[0], generator=torch.Generator().manual_seed(1)).to(torch.int32).view(seqs, -1).cuda()
    fx.cache_write(cache, table, torch.zeros(seqs, dtype=torch.int32, device="cuda"), k, v, seqs=fx.build_sequences(jo))
    out, _ = fx.attention_step(cache, table, torch.full((seqs,), n, dtype=torch.int32, device="cuda"), q)
    ro, _, bo, _ = _step_bounds(q64, held(k64), held(v64), bounds, dtype, store)
    A.check(_f64(out), ro, bo, dtype, "out")
