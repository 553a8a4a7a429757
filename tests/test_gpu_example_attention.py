"""The example network with an attention block: runs, every gradient reaches its weight and is the difference quotient; and its scenes
that grow row by row over a paged cache."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_it_runs_with_attention():
    import voxel_mixer as V
    net, losses = V.train(steps=3, heads=4, kv_heads=2)
    assert all(p.grad is not None and torch.isfinite(p.grad).all() and p.grad.any() for p in net.parameters())
    assert all(l == l for l in losses)
    net.eval()
    feat, maps, _ = V.scenes()
    assert torch.equal(net(feat, maps), net(feat, maps))


def test_gradients_through_the_attention_block():
    """Along one direction for each weight, in fp32 with dropout on, by a step of 2^-6 (1 in length) either side: third derivatives
    and sums of fp32 losses stay below two per cent of the directional derivative's scale."""
    import voxel_mixer as V
    feat, maps, target = V.scenes(dtype=torch.float32)
    net = V.VoxelMixer(feat.shape[1], c=32, heads=2)
    loss = lambda: (net(feat, maps, 7).double() - target).square().mean()
    loss().backward()
    gen = torch.Generator(device="cuda").manual_seed(9)
    for name in ("attend", "mix", "post3", "w3", "scale3"):
        p = getattr(net, name)
        d = torch.randn(p.shape, generator=gen, device="cuda")
        d /= d.norm()
        eps = 2.0 ** -6
        with torch.no_grad():
            p += eps * d
            up = float(loss())
            p -= 2 * eps * d
            down = float(loss())
            p += eps * d
        assert abs((up - down) / (2 * eps) - float((p.grad * d).sum())) <= 2e-2 * float(p.grad.norm()) + 1e-6, name


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_growing(dtype):
    import voxel_mixer as V
    got, whole = V.grow(rows=220, prompt=200, dtype=dtype)
    # A result is at most the largest value, the first rows' own.  bf16: the call's weights and both results are rounded by 2^-8.
    # fp32: a score of 64 products of some 5 in all is off by 66 * 5 * 2^-24 = 2e-5, weights by that and the sum's, on both sides.
    assert float((got.float() - whole.float()).abs().max()) <= (1e-4 if dtype == torch.float32 else 3 * 2.0 ** -8) * float(whole.abs().max())


def test_growing_over_8_bits():
    import voxel_mixer as V
    got, whole = V.grow(rows=220, prompt=200, store=torch.float8_e4m3fn)
    assert torch.equal(got[:, :200], V.grow(rows=220, prompt=200)[0][:, :200]) and torch.isfinite(got).all() and got.shape == whole.shape
