"""What stands in rows of a cache that no sequence sees: any bytes, in keys, values and exponents, add nothing to a step."""
import numpy as np
import pytest
import torch

import attention_reference as A
import paper_2407_01781_amd as fx
from test_gpu_attention import _f64, _held, _joff, draw

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,store,d", [("bf16", "e4m3", 64), ("f16", "e4m3", 16), ("f32", "e4m3", 128), ("bf16", "bf16", 32), ("f16", "f16", 64), ("f32", "f32", 48), ("bf16", "e4m3", 208)])
@pytest.mark.parametrize("fill", [0xFF, 0x7F, 0x7C, 0x80])
def test_rows_that_were_never_written(dtype, store, d, fill):
    lens, page, kvh, heads = [1, 5, 40, 700, 3000], 16, 2, 4
    bounds, jo = _joff(lens)
    need = [-(-n // page) for n in lens]
    pages = sum(need) + 3
    cache = fx.KVCache.empty(pages, page, kvh, d, torch.float8_e4m3fn if store == "e4m3" else {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}[store])
    for t in (cache.k, cache.v, cache.k_exp, cache.v_exp):
        if t is not None:
            t.view(torch.uint8).fill_(fill)
    order = np.random.default_rng(1).permutation(np.arange(1, pages))           # page 0 belongs to nobody
    table = np.full((len(lens), max(need) + 1), -1, np.int32)
    for b, n in enumerate(need):
        table[b, :n] = order[sum(need[:b]):sum(need[:b]) + n]
    table[3, 7] = -1                    # and one inside a sequence
    table = torch.from_numpy(table).cuda()
    (k, k64), (v, v64) = (draw(s, bounds[-1], kvh, d, dtype) for s in (1, 2))
    q, q64 = draw(3, len(lens), heads, d, dtype)
    fx.cache_write(cache, table, torch.zeros(len(lens), dtype=torch.int32, device="cuda"), k, v, seqs=fx.build_sequences(jo))
    out, lse = fx.attention_step(cache, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), q)
    there = np.ones(bounds[-1], bool)
    there[bounds[3] + 7 * page:bounds[3] + 8 * page] = False
    held = [_held(x, store)[there] for x in (k64, v64)]
    real = np.cumsum([0] + [int(there[a:b].sum()) for a, b in jo])
    ro, rl, bo, bl = A.attention(q64, *held, np.arange(len(lens) + 1), real, False, d ** -0.5, dtype)
    A.check(_f64(lse), rl.T, bl.T, "f32", "lse")
    A.check(_f64(out), ro, bo, dtype, "out")
