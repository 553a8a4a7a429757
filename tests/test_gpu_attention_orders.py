"""Inputs of attention that are broadcast, as the gradient of a sum is: the same bits as from a copy of their values."""
import pytest
import torch

import paper_2407_01781_amd as fx
from test_gpu_attention import _joff, draw

pytestmark = pytest.mark.gpu

LENS = [40, 0, 70, 1]


@pytest.mark.parametrize("which", range(4))
@pytest.mark.parametrize("dim", [None, 0, 1, 2])
def test_broadcast(which, dim):
    """One value for all, one row, one head or one element: as a loss that is a sum gives."""
    b, jo = _joff(LENS)
    seqs = fx.build_sequences(jo)
    t = [draw(s, b[-1], h, 64, "bf16")[0] for s, h in ((1, 4), (2, 4), (3, 4), (4, 4))]
    x = t[which]
    t[which] = (x[:1, :1, :1] if dim is None else x.narrow(dim, 0, 1)).expand_as(x)
    plain = [y.contiguous() for y in t]
    assert 0 in t[which].stride()
    out, lse = fx.attention_fwd(seqs, *plain[:3])
    for x, y in zip(fx.attention_fwd(seqs, *t[:3]), (out, lse)):
        assert torch.equal(x, y)
    for x, y in zip(fx.attention_bwd(seqs, *t[:3], out, lse, t[3]), fx.attention_bwd(seqs, *plain[:3], out, lse, plain[3])):
        assert torch.equal(x, y)


def test_a_sum_as_loss():
    from examples.voxel_mixer import Attention
    b, jo = _joff(LENS)
    seqs = fx.build_sequences(jo)
    packed = draw(1, b[-1], 1, 8 * 32, "f32")[0].view(int(b[-1]), -1).requires_grad_()
    Attention.apply(packed, seqs, 4, 2, True).sum().backward()
    got, packed.grad = packed.grad, None
    out = Attention.apply(packed, seqs, 4, 2, True)
    out.backward(torch.ones_like(out))
    assert torch.equal(got, packed.grad) and got.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_the_cache_and_the_step(dtype):
    d, n = 48, 5
    k, v, q = (draw(s, n, h, d, dtype)[0] for s, h in ((1, 2), (2, 2), (3, 4)))
    table, at = torch.arange(n, dtype=torch.int32, device="cuda")[:, None].contiguous(), torch.zeros(n, dtype=torch.int32, device="cuda")
    new = lambda: fx.KVCache.empty(n, 16, 2, d, k.dtype)
    ref = new()
    fx.cache_write(ref, table, at, k, v)
    cache, one = new(), new()
    fx.cache_write(cache, table, at, k[:1].expand_as(k), v[:, :1].expand_as(v))
    fx.cache_write(one, table, at, k[:1].expand_as(k).contiguous(), v[:, :1].expand_as(v).contiguous())
    assert torch.equal(cache.k, one.k) and torch.equal(cache.v, one.v)
    assert all(torch.equal(x, y) for x, y in zip(fx.attention_step(ref, table, at + 1, q[:1].expand_as(q)), fx.attention_step(ref, table, at + 1, q[:1].expand_as(q).contiguous())))


def test_orders_that_are_refused():
    """Outputs that are broadcast; elements of a head that lie apart."""
    b, jo = _joff(LENS)
    seqs = fx.build_sequences(jo)
    q, k, v = (draw(s, b[-1], h, 32, "f32")[0] for s, h in ((1, 4), (2, 2), (3, 2)))
    with pytest.raises(AssertionError, match="out"):
        fx.attention_fwd(seqs, q, k, v, out=torch.empty((q.shape[0], 32, 4), device="cuda").transpose(1, 2))
    with pytest.raises(AssertionError, match="out"):
        fx.attention_fwd(seqs, q, k, v, out=torch.empty((1, 4, 32), device="cuda").expand_as(q))
    with pytest.raises(AssertionError, match="v"):
        fx.attention_fwd(seqs, q, k, torch.empty((*v.shape[:2], 64), device="cuda")[..., ::2])
