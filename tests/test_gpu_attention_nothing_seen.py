"""Rows that see no key and keys that no row gives a weight: gradients of zero, whatever else stands there."""
import numpy as np
import pytest
import torch

import attention_reference as A
import paper_2407_01781_amd as fx
from test_gpu_attention import _f64, _joff, draw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,kv_lens,heads,kv_heads,d,dtype", [([70], [40], 2, 1, 64, "bf16"), ([12, 9, 30], [3, 0, 29], 2, 2, 32, "f16"), ([300, 5], [200, 9], 4, 2, 128, "f16"), ([90], [1], 1, 1, 40, "f32"),
                                                                 ([2500], [2300], 8, 8, 64, "bf16"), ([200] * 30, [150] * 30, 4, 4, 32, "f32"), ([330], [300], 1, 1, 200, "bf16")])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_rows_that_see_no_key(lens, kv_lens, heads, kv_heads, d, dtype, bad):
    bq, jq = _joff(lens)
    bk, jk = _joff(kv_lens)
    seqs, kv = fx.build_sequences(jq), fx.build_sequences(jk)
    q, k, v, go = (draw(s, m, h, d, dtype)[0] for s, m, h in ((1, bq[-1], heads), (2, bk[-1], kv_heads), (3, bk[-1], kv_heads), (4, bq[-1], heads)))
    gl = torch.from_numpy(np.random.default_rng(5).standard_normal((heads, int(bq[-1]))).astype(np.float32)).cuda()
    out, lse = fx.attention_fwd(seqs, q, k, v, causal=True, kv_seqs=kv)
    ref = fx.attention_bwd(seqs, q, k, v, out, lse, go, grad_lse=gl, causal=True, kv_seqs=kv)
    alone = np.concatenate([np.arange(bq[s], bq[s] + max(0, n - m)) for s, (n, m) in enumerate(zip(lens, kv_lens))])
    assert torch.isneginf(lse[:, alone]).all() and not out[alone].any() and not ref[0][alone].any()
    for r in alone[[0, len(alone) // 2, -1]]:
        go[r, -1, d // 2] = bad
    for r in alone[[0, len(alone) // 3, -1]]:
        gl[0, r] = bad
    q[alone[-1], 0, 0] = bad
    got = fx.attention_bwd(seqs, q, k, v, out, lse, go, grad_lse=gl, causal=True, kv_seqs=kv)
    assert not got[0][alone].any()
    assert all(torch.equal(x, y) for x, y in zip(got, ref))


@pytest.mark.parametrize("lens,heads,kv_heads,d,dtype", [([40, 70], 2, 1, 64, "bf16"), ([5], 2, 2, 32, "f16"), ([300], 4, 2, 128, "f16"), ([33, 7], 1, 1, 40, "f32"), ([1000, 900], 8, 8, 64, "bf16"),
                                                         ([45] * 30, 4, 4, 32, "f32"), ([330], 1, 1, 200, "bf16")])
@pytest.mark.parametrize("causal", [False, True])
def test_keys_that_no_row_weighs(lens, heads, kv_heads, d, dtype, causal):
    """Keys of which one element is -inf, where every query has 1: scores of -inf.  Out and all gradients but gq's in that channel are those
    without these keys (gq has 0 times -inf there)."""
    b, jo = _joff(lens)
    n = int(b[-1])
    seqs, s = fx.build_sequences(jo), d ** -0.5
    t = [draw(i, n, h, d, dtype)[0] for i, h in ((1, heads), (2, kv_heads), (3, kv_heads), (4, heads))]
    q, k, v, go = t
    q[:, :, 0] = 1
    gone = np.unique(np.concatenate([b[:-1] + 2, b[1:] - 2, b[:-1] + (b[1:] - b[:-1]) // 2]))
    k[torch.from_numpy(gone).cuda(), :, 0] = float("-inf")
    out, lse = fx.attention_fwd(seqs, q, k, v, causal=causal)
    got = [_f64(x) for x in fx.attention_bwd(seqs, q, k, v, out, lse, go, causal=causal)]
    f = [_f64(x) for x in t]
    f[1][gone, :, 0] = -1e6             # for the formulas: weights of 0 all the same
    ro, rl, bo, bl = A.attention(*f[:3], b, b, causal, s, dtype)
    ref = A.attention_grad(*f, b, b, causal, s, dtype)
    live = ro[:, :, 0] != 0             # a causal row that sees such keys alone has scores of -inf and no others
    A.check(_f64(out)[live], ro[live], bo[live], dtype, "out")
    A.check(got[0][live][:, 1:], ref[0][live][:, 1:], ref[3][live][:, 1:], dtype, "gq")
    for i in (1, 2):
        assert not got[i][gone].any(), f"gradient {i} of keys without weight"
        A.check(got[i], ref[i], ref[3 + i], dtype, f"gradient {i}")
