"""A small network on voxels, trained and then run on a stream of them: a convolution block and a recurrence block around
one residual stream, from this library's operators with their gradients.

    x      = dropout(conv3(features))
    x, n   = join(x, conv3(norm(x)), gate = conv1(norm(x)))           a convolution's reach: 3 x 3 x 3 voxels
    u | z  = conv1(n)
    x, n   = join(x, scan(u, z) + scan(u, z, reversed))               along all voxels of a scene, in index order
    result = n . head

``python examples/voxel_mixer.py`` prints the loss of a few steps on indoor-like scenes (the target: how full a voxel's
surroundings are, and how far along the scene it lies, which no 3 x 3 x 3 stencil can know).
"""
from __future__ import annotations

import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2407_01781_amd as fx  # noqa: E402
from workloads import generators as G  # noqa: E402


# ------------------------------------------------------------------------------------------ the operators as torch functions
class Conv(torch.autograd.Function):
    """Sparse convolution over a kernel map (1x1x1: a product with the features)."""

    @staticmethod
    def forward(ctx, x, w, kmap):
        ctx.kmap, ctx.dt = kmap, w.dtype
        w = w.to(x.dtype)
        ctx.save_for_backward(x, w)
        return fx.sparse_conv_fwd(kmap, x, w)

    @staticmethod
    def backward(ctx, g):
        x, w = ctx.saved_tensors
        g = g.contiguous()
        gx = fx.sparse_conv_bwd_data(ctx.kmap, g, w) if ctx.needs_input_grad[0] else None
        return gx, fx.sparse_conv_bwd_weight(ctx.kmap, x, g, out_dtype=torch.float32).to(ctx.dt), None


class Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w):
        ctx.save_for_backward(x, w)
        return fx.rms_norm_fwd(x, w)

    @staticmethod
    def backward(ctx, g):
        return fx.rms_norm_bwd(g, *ctx.saved_tensors)


class Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, *mask):
        ctx.mask = mask
        return fx.dropout(x, *mask)

    @staticmethod
    def backward(ctx, g):
        return fx.dropout(g, *ctx.mask), None, None, None


class Scan(torch.autograd.Function):
    """Takes the features and the gate as they come out of one projection [N, 2C]."""

    @staticmethod
    def forward(ctx, both, seqs, reverse):
        u, z = both.chunk(2, 1)
        h, _ = fx.gated_scan_fwd(seqs, u, z, reverse=reverse)
        ctx.seqs, ctx.reverse = seqs, reverse
        ctx.save_for_backward(both, h)
        return h

    @staticmethod
    def backward(ctx, g):
        both, h = ctx.saved_tensors
        u, z = both.chunk(2, 1)
        gu, gz, _ = fx.gated_scan_bwd(ctx.seqs, u, z, h, g, reverse=ctx.reverse)
        return torch.cat([gu, gz], 1), None, None


class Join(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, y, gate, post, scale, nxt, p, seed, offset):
        ctx.kw = dict(act="silu", p=p, seed=seed, offset=offset)
        out, n = fx.block_join_fwd(x, y, gate=gate, post_weight=post, scale=scale, next_weight=nxt, **ctx.kw)
        ctx.save_for_backward(out, y, gate, post, scale, nxt)
        return out, n

    @staticmethod
    def backward(ctx, g_out, g_norm):
        out, y, gate, post, scale, nxt = ctx.saved_tensors
        g = fx.block_join_bwd(g_out, g_norm, out, y, gate=gate, post_weight=post, scale=scale, next_weight=nxt, **ctx.kw)
        return g["x"], g["y"], g["gate"], g["post"], g["scale"], g["next"], None, None, None


# ------------------------------------------------------------------------------------------ the network
class VoxelMixer(torch.nn.Module):
    def __init__(self, c_in=8, c=64, p=0.1, seed=1):
        super().__init__()
        gen = torch.Generator().manual_seed(seed)
        def weight(*shape):
            return torch.nn.Parameter((torch.randn(shape, generator=gen) * (shape[0] * shape[1]) ** -0.5).cuda())
        def ones(v=1.0):
            return torch.nn.Parameter(torch.full((c,), v, device="cuda"))
        self.stem, self.conv, self.gate = weight(27, c_in, c), weight(27, c, c), weight(1, c, c)
        self.project, self.head = weight(1, c, 2 * c), weight(1, c, 2)
        self.w1, self.post1, self.scale1, self.w2 = ones(), ones(), ones(0.5), ones()
        self.post2, self.scale2, self.w3 = ones(), ones(0.5), ones()
        # the first of the gate's channels forget within a few rows, the last remember for some thousand
        self.memory = torch.nn.Parameter(torch.linspace(-1.0, 7.0, c, device="cuda"))
        self.p, self.seed = p, seed

    def forward(self, feat, grid_maps, step=0):
        k3, k1, seqs = grid_maps
        p = self.p if self.training else 0.0
        mask = lambda i: (p, self.seed, 4 * step + i)           # every call's mask has an offset of its own
        x = Dropout.apply(Conv.apply(feat, self.stem, k3), *mask(0))
        n = Norm.apply(x, self.w1)
        x, n = Join.apply(x, Conv.apply(n, self.conv, k3), Conv.apply(n, self.gate, k1), self.post1, self.scale1, self.w2, *mask(1))
        both = Conv.apply(n, self.project, k1)
        both = torch.cat([both[:, :both.shape[1] // 2], both[:, both.shape[1] // 2:] + self.memory.to(both.dtype)], 1)
        y = Scan.apply(both, seqs, False) + Scan.apply(both, seqs, True)
        x, n = Join.apply(x, y, None, self.post2, self.scale2, self.w3, *mask(2))
        return Conv.apply(n, self.head, k1)


def scenes(name="indoor_small", dtype=torch.bfloat16):
    """A batch of grids with its maps, input features and targets."""
    w = G.workload(name)
    ijk, jo = w.jagged_ijk()
    grid = fx.build_index_grid(torch.from_numpy(ijk).cuda(), jo)
    maps = (fx.build_kernel_map(grid, 3, 1), fx.build_kernel_map(grid, 1, 1), fx.build_sequences(grid.voxel_joffsets()))
    n = grid.num_voxels
    full = (maps[0].dense() >= 0).sum(1, keepdim=True).float() / 27
    along = torch.cat([torch.linspace(-1, 1, int(b - a)) for a, b in grid.voxel_joffsets()])[:, None].cuda()
    gen = torch.Generator(device="cuda").manual_seed(3)
    feat = torch.cat([torch.ones((n, 1), device="cuda"), torch.randn((n, 7), generator=gen, device="cuda")], 1).to(dtype)
    return feat, maps, torch.cat([full, along], 1)


def train(steps=40, lr=3e-3, name="indoor_small", dtype=torch.bfloat16, report=None):
    feat, maps, target = scenes(name, dtype)
    net = VoxelMixer(feat.shape[1])
    opt = torch.optim.Adam(net.parameters(), lr=lr)
    losses = []
    for step in range(steps):
        loss = (net(feat, maps, step).float() - target).square().mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(float(loss.detach()))
        if report and step % 10 == 0:
            report(f"step {step}: loss {losses[-1]:.4f}")
    return net, losses


def stream(rows=1_000, c=64, chunk=300):
    """A scan that arrives in parts: the state behind a part goes into the next one, single rows at the end.  Returns the
    rows and what one call over all of them gives."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    u, z = (torch.randn((rows, c), generator=gen, device="cuda") + b for b in (0.0, 2.0))
    whole, _ = fx.gated_scan_fwd(fx.build_sequences([[0, rows]]), u, z)
    state, parts = torch.zeros((1, c), device="cuda"), []
    at = 0
    while at + chunk <= rows:
        h, state = fx.gated_scan_fwd(fx.build_sequences([[0, chunk]]), u[at:at + chunk], z[at:at + chunk], h0=state)
        parts.append(h)
        at += chunk
    for r in range(at, rows):
        h, state = fx.gated_scan_step(u[r:r + 1], z[r:r + 1], state, new_state=state)
        parts.append(h)
    return torch.cat(parts), whole


if __name__ == "__main__":
    _, losses = train(report=print)
    print(f"loss {losses[0]:.4f} -> {np.mean(losses[-5:]):.4f}")
    got, whole = stream()
    print(f"streamed rows against one call: {float((got - whole).abs().max()):.1e}")
