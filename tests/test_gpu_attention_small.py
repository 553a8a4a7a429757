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
    """Weights of some 2^-18: what the kernels lose of one is 2^-40 at most, and of a gradient of a score 2^-36 of its row's largest, here 2^-10."""
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
