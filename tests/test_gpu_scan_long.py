"""The recurrence over many tiles against the formulas in 64 bits, row by row: more groups of tiles than one looks back over,
states that live across them, sequences that begin inside a group far before the end, more channels than a slab has.

Rows a tile has (a workgroup's threads, 16 lanes a row at 64 channels, rows a lane): 256 forward and with gradients of a
16-bit type, 128 with gradients of f32, where a workgroup has 512 threads, which it has from 16 tiles (of all slabs) on;
2048 at 8 channels.  16 tiles are a group, 16 groups are looked back over at a time."""
import numpy as np
import pytest
import torch

import gpu_common as H
import paper_2407_01781_amd as fx
import rows_reference as R
import test_gpu_scan as T

pytestmark = pytest.mark.gpu


def _one(lens, c, dtype, reverse, seed, packed=False):
    """Forward and gradients with states handed in.  The gates' biases run over the channels: the first forget within a few
    rows, the last remember for some ten thousand; inputs and gradients have a mean, which long memory adds up."""
    bounds, jo = T._joff(lens)
    n, b = int(bounds[-1]), len(lens)
    seqs = fx.build_sequences(jo)
    bias = np.linspace(-1.0, 9.0, c)
    x, rx = T._draw(seed, n, c, dtype, packed, mean=1.0)
    z, rz = T._draw(seed + 1, n, c, dtype, packed, mean=bias)
    gh, rgh = T._draw(seed + 2, n, c, dtype, packed, mean=0.25)
    s0, r0 = T._draw(seed + 3, b, c, "f32", std=4.0)
    gl, rgl = T._draw(seed + 4, b, c, "f32", std=100.0)
    out = H.nan_filled((n, c), x.dtype)
    h, last = fx.gated_scan_fwd(seqs, x, z, h0=s0, reverse=reverse, out=out)
    ref, rlast, E, El = R.scan(rx, rz, bounds, r0, reverse)
    R.check(T._f64(h), ref, E, dtype, "h")
    R.check(T._f64(last), rlast, El, "f32", "last")
    gx, gz, g0 = fx.gated_scan_bwd(seqs, x, z, h, gh, h0=s0, grad_last=gl, reverse=reverse)
    want = R.scan_grad(rx, rz, T._f64(h), rgh, bounds, r0, rgl, reverse)
    R.check(T._f64(gx), want[0], want[3], dtype, "gx")
    R.check(T._f64(gz), want[1], want[4], dtype, "ggate")
    R.check(T._f64(g0), want[2], want[5], "f32", "gh0")


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_sequence(dtype, reverse):
    _one([100_003], 64, dtype, reverse, 101)            # 391 tiles and 25 groups; gradients of f32 782 and 49


@pytest.mark.parametrize("reverse", [False, True])
def test_sequences_that_begin_inside_a_group(reverse):
    # seven and a half tiles into the first group; then one of 20 groups, and single rows between long ones
    _one([1_921, 81_920, 1, 0, 1, 6_000], 64, "f16", reverse, 111)


@pytest.mark.parametrize("reverse", [False, True])
def test_slabs(reverse):
    _one([77_777], 137, "f32", reverse, 121)            # three slabs, the last of nine channels: 304 tiles each, 608 with gradients


def test_few_channels():
    _one([150_000], 3, "bf16", False, 131, packed=True)     # one lane a row, 4096 rows a tile


# forward and gradients of a 16-bit type: one tile, at its edge; the fewest tiles of 512 threads; a group and two of them
EDGES = [255, 256, 257, 4_095, 4_096, 4_097, 8_191, 8_192, 8_193]


@pytest.mark.parametrize("rows", EDGES)
@pytest.mark.parametrize("reverse", [False, True])
def test_edges_of_tiles_and_groups(rows, reverse):
    _one([rows], 64, "bf16", reverse, 141)


@pytest.mark.parametrize("rows", [127, 128, 129, 2_047, 2_048, 2_049, 4_097])
@pytest.mark.parametrize("reverse", [False, True])
def test_edges_of_tiles_and_groups_with_gradients_of_f32(rows, reverse):
    _one([rows], 64, "f32", reverse, 151)


@pytest.mark.parametrize("reverse", [False, True])
def test_sequences_that_begin_with_a_tile(reverse):
    # with the first tile of a group, with the last, with one inside; counted from either end
    _one([4_096, 3_840, 256, 1_024, 3_072, 4_096], 64, "bf16", reverse, 161)


def test_edges_at_few_channels():
    for rows in (32_767, 32_768, 32_769):               # 16 tiles of 2048 rows
        _one([rows], 8, "bf16", False, 171)
