"""A small network on voxels, trained and then run on a stream of them: a convolution block and a recurrence block around
one residual stream, from this library's operators with their gradients.

    x      = dropout(conv3(features))
    x, n   = join(x, conv3(norm(x)), gate = conv1(norm(x)))           a convolution's reach: 3 x 3 x 3 voxels
    u | z  = conv1(n)
    x, n   = join(x, scan(u, z) + scan(u, z, reversed))               along all voxels of a scene, in index order
    x, n   = join(x, conv1(attention(conv1(n))))                      inside windows of 512 voxels; with heads, left out without
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


class Attention(torch.autograd.Function):
    """Takes queries, keys and values as they come out of one projection [N, (heads + 2 kv_heads) dim]."""

    @staticmethod
    def forward(ctx, packed, seqs, heads, kv_heads, causal):
        q, k, v = packed.view(packed.shape[0], heads + 2 * kv_heads, -1).split([heads, kv_heads, kv_heads], 1)
        out, lse = fx.attention_fwd(seqs, q, k, v, causal=causal)
        ctx.args = seqs, heads, kv_heads, causal
        ctx.save_for_backward(packed, out, lse)
        return out.flatten(1)

    @staticmethod
    def backward(ctx, g):
        packed, out, lse = ctx.saved_tensors
        seqs, heads, kv_heads, causal = ctx.args
        q, k, v = packed.view(packed.shape[0], heads + 2 * kv_heads, -1).split([heads, kv_heads, kv_heads], 1)
        grads = fx.attention_bwd(seqs, q, k, v, out, lse, g.reshape(out.shape), causal=causal)
        return torch.cat(grads, 1).flatten(1), None, None, None, None


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
    def __init__(self, c_in=8, c=64, p=0.1, seed=1, heads=0, kv_heads=0):
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
        self.p, self.seed, self.heads, self.kv_heads = p, seed, heads, kv_heads or heads
        if heads:
            self.attend = weight(1, c, (heads + 2 * self.kv_heads) * (c // heads))
            self.mix, self.post3, self.scale3, self.w4 = weight(1, c, c), ones(), ones(0.5), ones()

    def forward(self, feat, grid_maps, step=0):
        k3, k1, seqs, near = grid_maps
        p = self.p if self.training else 0.0
        mask = lambda i: (p, self.seed, 4 * step + i)           # every call's mask has an offset of its own (four a step)
        x = Dropout.apply(Conv.apply(feat, self.stem, k3), *mask(0))
        n = Norm.apply(x, self.w1)
        x, n = Join.apply(x, Conv.apply(n, self.conv, k3), Conv.apply(n, self.gate, k1), self.post1, self.scale1, self.w2, *mask(1))
        both = Conv.apply(n, self.project, k1)
        both = torch.cat([both[:, :both.shape[1] // 2], both[:, both.shape[1] // 2:] + self.memory.to(both.dtype)], 1)
        y = Scan.apply(both, seqs, False) + Scan.apply(both, seqs, True)
        x, n = Join.apply(x, y, None, self.post2, self.scale2, self.w3, *mask(2))
        if self.heads:
            y = Attention.apply(Conv.apply(n, self.attend, k1), near, self.heads, self.kv_heads, False)
            x, n = Join.apply(x, Conv.apply(y, self.mix, k1), None, self.post3, self.scale3, self.w4, *mask(3))
        return Conv.apply(n, self.head, k1)


def windows(joffsets, size=512):
    """Ranges of up to `size` rows of every range, in order."""
    parts = [np.arange(a, b, size) for a, b in joffsets]
    first = np.concatenate(parts) if parts else np.zeros(0, np.int64)
    end = np.concatenate([np.minimum(p + size, b) for p, (_, b) in zip(parts, joffsets)]) if parts else first
    return np.stack([first, end], 1)


def scenes(name="indoor_small", dtype=torch.bfloat16):
    """A batch of grids with its maps, input features and targets."""
    w = G.workload(name)
    ijk, jo = w.jagged_ijk()
    grid = fx.build_index_grid(torch.from_numpy(ijk).cuda(), jo)
    maps = (fx.build_kernel_map(grid, 3, 1), fx.build_kernel_map(grid, 1, 1), fx.build_sequences(grid.voxel_joffsets()),
            fx.build_sequences(windows(grid.voxel_joffsets())))
    n = grid.num_voxels
    full = (maps[0].dense() >= 0).sum(1, keepdim=True).float() / 27
    along = torch.cat([torch.linspace(-1, 1, int(b - a)) for a, b in grid.voxel_joffsets()])[:, None].cuda()
    gen = torch.Generator(device="cuda").manual_seed(3)
    feat = torch.cat([torch.ones((n, 1), device="cuda"), torch.randn((n, 7), generator=gen, device="cuda")], 1).to(dtype)
    return feat, maps, torch.cat([full, along], 1)


def train(steps=40, lr=3e-3, name="indoor_small", dtype=torch.bfloat16, report=None, heads=0, kv_heads=0):
    feat, maps, target = scenes(name, dtype)
    net = VoxelMixer(feat.shape[1], heads=heads, kv_heads=kv_heads)
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


def grow(rows=700, prompt=600, heads=8, kv_heads=2, d=64, page=16, dtype=torch.bfloat16, store=None, seqs=3):
    """Scenes that grow row by row: attention inside what is there, its keys and values into a paged cache (of `store`, 8 bits
    say), then one new row of each scene at a time.  Returns the rows and what one causal call over all of them gives."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    q, k, v = (torch.randn((seqs, rows, h, d), generator=gen, device="cuda").to(dtype) for h in (heads, kv_heads, kv_heads))
    ranges = lambda n: [[s * n, (s + 1) * n] for s in range(seqs)]
    whole, _ = fx.attention_fwd(fx.build_sequences(ranges(rows)), q.flatten(0, 1), k.flatten(0, 1), v.flatten(0, 1), causal=True)
    columns = -(-rows // page)
    cache = fx.KVCache.empty(seqs * columns, page, kv_heads, d, store or dtype)
    table = torch.randperm(seqs * columns, generator=gen, device="cuda").to(torch.int32).view(seqs, columns)
    lengths = torch.zeros(seqs, dtype=torch.int32, device="cuda")
    first = fx.build_sequences(ranges(prompt))
    out, _ = fx.attention_fwd(first, q[:, :prompt].flatten(0, 1), k[:, :prompt].flatten(0, 1), v[:, :prompt].flatten(0, 1), causal=True)
    fx.cache_write(cache, table, lengths, k[:, :prompt].flatten(0, 1), v[:, :prompt].flatten(0, 1), seqs=first)
    lengths += prompt
    parts = [out.view(seqs, prompt, heads, d)]
    for r in range(prompt, rows):
        fx.cache_write(cache, table, lengths, k[:, r], v[:, r])
        lengths += 1
        parts.append(fx.attention_step(cache, table, lengths, q[:, r])[0][:, None])
    return torch.cat(parts, 1), whole.view(seqs, rows, heads, d)


if __name__ == "__main__":
    _, losses = train(report=print)
    print(f"loss {losses[0]:.4f} -> {np.mean(losses[-5:]):.4f}")
    got, whole = stream()
    print(f"streamed rows against one call: {float((got - whole).abs().max()):.1e}")
    for store in (None, torch.float8_e4m3fn):
        got, whole = grow(store=store)
        print(f"rows over a cache of {store or 'their own type'} against one causal call: {float((got - whole).abs().max()):.1e}")
