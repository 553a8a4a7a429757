"""The example network: trains (every gradient reaches its weight and the loss falls), evaluates without dropout the same
every time, and its recurrence runs in parts as it does in one call."""
import os
import sys

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_it_trains():
    import voxel_mixer as V
    net, losses = V.train(steps=30)
    assert all(p.grad is not None and torch.isfinite(p.grad).all() and p.grad.any() for p in net.parameters())
    # the target's two columns have a mean square of about 0.2 and 1/3: predicting nothing is the first loss at least
    assert np.mean(losses[-5:]) <= 0.5 * losses[0]
    net.eval()
    feat, maps, _ = V.scenes()
    assert torch.equal(net(feat, maps), net(feat, maps))


def test_weight_gradients_are_the_differences():
    """Along one direction per vector, in fp32 with dropout on, by a step of 2^-6 either side: third derivatives and sums of
    fp32 losses stay below two per cent of the directional derivative's scale."""
    import voxel_mixer as V
    feat, maps, target = V.scenes(dtype=torch.float32)
    net = V.VoxelMixer(feat.shape[1], c=32)
    loss = lambda: (net(feat, maps, 7).double() - target).square().mean()
    loss().backward()
    gen = torch.Generator(device="cuda").manual_seed(9)
    for name in ("w1", "post1", "scale1", "w2", "post2", "scale2", "w3", "memory"):
        p = getattr(net, name)
        d = torch.randn(p.shape, generator=gen, device="cuda")
        eps = 2.0 ** -6
        with torch.no_grad():
            p += eps * d
            up = float(loss())
            p -= 2 * eps * d
            down = float(loss())
            p += eps * d
        assert abs((up - down) / (2 * eps) - float((p.grad * d).sum())) <= 2e-2 * float(p.grad.norm()) * float(d.norm()) + 1e-6, name


def test_streaming():
    import voxel_mixer as V
    got, whole = V.stream()
    # the recurrence's own bound at gates up to 2 + 4 standard deviations: some 20 units a step over some 400 steps of memory
    assert float((got - whole).abs().max()) <= 400 * 20 * 2.0 ** -24 * 4
