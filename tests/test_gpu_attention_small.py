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
