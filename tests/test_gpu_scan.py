"""GPU parity of the gated linear recurrence: forward, gradients and single steps against the formulas in 64 bits, row
by row, at lengths around a lane's rows (8) and of up to some thirty tiles (the lengths named after a tile are from tiles
of 512 rows; today one has 32 there, and test_gpu_scan_long.py tests the edges); sequences without rows; every type; column
ranges of wider tensors; infinities and NaN; streams."""
import numpy as np
import pytest
import torch

import gpu_common as H
import paper_2407_01781_amd as fx
import rows_reference as R

pytestmark = pytest.mark.gpu


def _joff(lens):
    b = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
    return b, np.stack([b[:-1], b[1:]], 1)


def _draw(seed, n, c, dtype, packed=False, std=1.0, mean=0.0):
    """A tensor of rows, or its columns 1 .. c of a wider one; and the stored values in 64 bits."""
    rng = np.random.default_rng(seed)
    v = torch.from_numpy((rng.standard_normal((n, c)) * std + mean).astype(np.float32)).to(H.TORCH_DT[dtype])
    if packed:
        wide = torch.full((n, c + 4), 7.0, dtype=v.dtype, device="cuda")
        wide[:, 1:c + 1] = v.cuda()
        d = wide[:, 1:c + 1]
    else:
        d = v.cuda()
    return d, v.double().numpy()


def _f64(t):
    return t.double().cpu().numpy()


LENS = {
    "one row": [1], "one lane": [8], "nine": [9], "a tile less one": [511], "a tile": [512], "a tile and one": [513],
    "many tiles": [3001], "ragged": [0, 3, 1, 0, 0, 700, 2, 64, 8, 8, 1, 513, 0], "singles": [1] * 70, "none": [0, 0, 0], "no sequence": [],
}


@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("dtype,c", [("bf16", 64), ("f32", 5), ("f16", 33)])
def test_lengths(lens, reverse, dtype, c):
    _one(LENS[lens], c, dtype, reverse, h0=True, packed=False)


@pytest.mark.parametrize("c", [1, 2, 3, 4, 7, 8, 9, 15, 16, 17, 31, 63, 65, 100, 128, 137])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_channel_counts_and_column_ranges(c, dtype):
    _one([300, 0, 777], c, dtype, reverse=c % 2 == 0, h0=c % 3 == 0, packed=c % 4 != 0)


def test_many_tiles_of_few_channels():
    _one([9_000, 20_000], 6, "f32", False, h0=True, packed=True)


def _one(lens, c, dtype, reverse, h0, packed):
    bounds, jo = _joff(lens)
    n, b = int(bounds[-1]), len(lens)
    seqs = fx.build_sequences(jo)
    assert seqs.rows == n and seqs.batch_size == b
    x, rx = _draw(1, n, c, dtype, packed)
    z, rz = _draw(2, n, c, dtype, packed, std=2.0, mean=1.0)
    gh, rgh = _draw(3, n, c, dtype, packed)
    s0, r0 = _draw(4, b, c, "f32")
    gl, rgl = _draw(5, b, c, "f32")
    if not h0:
        s0 = r0 = gl = rgl = None
    out = H.nan_filled((n, c), x.dtype)
    h, last = fx.gated_scan_fwd(seqs, x, z, h0=s0, reverse=reverse, out=out)
    ref, rlast, E, El = R.scan(rx, rz, bounds, r0, reverse)
    R.check(_f64(h), ref, E, dtype, "h")
    R.check(_f64(last), rlast, El, "f32", "last")
    # the states as the forward call rounded them
    gx, gz, g0 = fx.gated_scan_bwd(seqs, x, z, h, gh, h0=s0, grad_last=gl, reverse=reverse)
    want = R.scan_grad(rx, rz, _f64(h), rgh, bounds, r0, rgl, reverse)
    R.check(_f64(gx), want[0], want[3], dtype, "gx")
    R.check(_f64(gz), want[1], want[4], dtype, "ggate")
    R.check(_f64(g0), want[2], want[5], "f32", "gh0")
    again = fx.gated_scan_bwd(seqs, x, z, h, gh, h0=s0, grad_last=gl, reverse=reverse)
    assert all(torch.equal(a, b) for a, b in zip((gx, gz, g0), again))


def test_gates_far_from_zero():
    """Gates that keep a state for thousands of rows, or nothing of it, and beyond the exponential's range."""
    n, c = 4_000, 16
    bounds, jo = _joff([n])
    x, rx = _draw(11, n, c, "f32")
    z, rz = _draw(12, n, c, "f32", std=0.5)
    shift = torch.tensor([0, 3, 6, 8, 10, 12, 20, 100, -3, -8, -20, -90, -200, 88, -88, 1e30])
    z += shift.cuda()
    rz = z.double().cpu().numpy()
    h, last = fx.gated_scan_fwd(fx.build_sequences(jo), x, z)
    ref, rlast, E, El = R.scan(rx, rz, bounds)
    R.check(_f64(h), ref, E, "f32")
    R.check(_f64(last), rlast, El, "f32")


def test_gradient_is_the_difference():
    """The derivative of a weighted sum of the outputs along one direction.  The difference over a step of 2^-7 either
    side is off by the third derivative (some 1e-4 of the whole at these gates) and by the rounding of sums of 3e3 terms
    of size one, 2^-24 x 3e3 / 2^-6; half a per cent covers both."""
    n, c = 200, 16
    bounds, jo = _joff([120, 80])
    seqs = fx.build_sequences(jo)
    (x, _), (z, _), (gh, _), (dx, _), (dz, _) = (_draw(s, n, c, "f32") for s in (21, 22, 23, 24, 25))
    loss = lambda x, z: float((fx.gated_scan_fwd(seqs, x, z)[0].double() * gh.double()).sum())
    h = fx.gated_scan_fwd(seqs, x, z)[0]
    gx, gz, _ = fx.gated_scan_bwd(seqs, x, z, h, gh)
    eps = 2.0 ** -7
    for g, d, (a, b) in ((gx, dx, (eps, 0)), (gz, dz, (0, eps))):
        num = (loss(x + a * dx, z + b * dz) - loss(x - a * dx, z - b * dz)) / (2 * eps)
        assert abs(num - float((g.double() * d.double()).sum())) <= 5e-3 * float((g.double() * d.double()).norm())


def test_a_sequence_in_two_calls():
    """The state behind the first part, handed to the second, gives the whole sequence's rows; single steps too."""
    n, c, cut = 1_500, 24, 1_111
    x, rx = _draw(31, n, c, "bf16")
    z, rz = _draw(32, n, c, "bf16", std=2.0)
    ref, rlast, E, El = R.scan(rx, rz, [0, n])
    h1, s = fx.gated_scan_fwd(fx.build_sequences([[0, cut]]), x[:cut], z[:cut])
    h2, s = fx.gated_scan_fwd(fx.build_sequences([[0, n - 5 - cut]]), x[cut:n - 5], z[cut:n - 5], h0=s)
    rows = [h1, h2]
    for t in range(n - 5, n):
        h, s = fx.gated_scan_step(x[t:t + 1], z[t:t + 1], s)
        rows.append(h)
    R.check(_f64(torch.cat(rows)), ref, E, "bf16")
    R.check(_f64(s), rlast, El, "f32")


@pytest.mark.parametrize("rows,c,dtype,packed", [(1, 1, "f32", False), (8, 256, "bf16", False), (3, 45, "f16", True), (700, 6, "bf16", True)])
def test_steps(rows, c, dtype, packed):
    x, rx = _draw(41, rows, c, dtype, packed)
    z, rz = _draw(42, rows, c, dtype, packed)
    s, rs = _draw(43, rows, c, "f32")
    ref, rlast, E, El = R.scan(rx, rz, np.arange(rows + 1), rs)
    h, new = fx.gated_scan_step(x, z, s)
    R.check(_f64(h), ref, E, dtype)
    R.check(_f64(new), rlast, El, "f32")
    h2, same = fx.gated_scan_step(x, z, s, new_state=s)
    assert same is s and torch.equal(h2, h) and torch.equal(s, new)


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("reverse", [False, True])
def test_what_is_not_finite_stays_in_its_sequence_and_channel(bad, reverse):
    lens = [40, 700, 9, 1200, 1, 600]
    bounds, jo = _joff(lens)
    n, c = int(bounds[-1]), 40
    seqs = fx.build_sequences(jo)
    x, _ = _draw(51, n, c, "f32")
    z, _ = _draw(52, n, c, "f32")
    gh, _ = _draw(53, n, c, "f32")
    clean = fx.gated_scan_fwd(seqs, x, z, reverse=reverse)
    clean_g = fx.gated_scan_bwd(seqs, x, z, clean[0], gh, reverse=reverse)
    at = int(bounds[3]) + 640
    x2, z2, gh2 = x.clone(), z.clone(), gh.clone()
    x2[at, 3] = bad
    z2[at, 17] = float("nan")
    got = fx.gated_scan_fwd(seqs, x2, z2, reverse=reverse)
    touched = torch.zeros((n, c), dtype=torch.bool, device="cuda")
    rows = slice(int(bounds[3]), at + 1) if reverse else slice(at, int(bounds[4]))
    touched[rows, 3] = touched[rows, 17] = True
    assert torch.equal(got[0][~touched], clean[0][~touched]) and not torch.isfinite(got[0][touched]).any()
    gh2[at, 5] = bad
    got = fx.gated_scan_bwd(seqs, x, z, clean[0], gh2, reverse=reverse)
    touched[:] = False
    touched[slice(at, int(bounds[4])) if reverse else slice(int(bounds[3]), at + 1), 5] = True
    for a, b in zip(got[:2], clean_g[:2]):
        assert torch.equal(a[~touched], b[~touched])
    assert not torch.isfinite(got[0][touched]).any()


def test_offsets_beyond_32_bits():
    """Rows so far apart that the last lie more than 2^32 bytes from the first."""
    n, c, ld = 5_000, 64, 500_000
    wide = torch.empty(n * ld, dtype=torch.bfloat16, device="cuda")
    x, z = wide.as_strided((n, c), (ld, 1), 0), wide.as_strided((n, c), (ld, 1), 1_000)
    small = [_draw(s, n, c, "bf16")[0] for s in (61, 62, 63)]
    x.copy_(small[0])
    z.copy_(small[1])
    seqs = fx.build_sequences([[0, 10], [10, n]])
    out = wide.as_strided((n, c), (ld, 1), 2_000)
    h, last = fx.gated_scan_fwd(seqs, x, z, out=out)
    h2, last2 = fx.gated_scan_fwd(seqs, small[0], small[1])
    assert torch.equal(h, h2) and torch.equal(last, last2)
    for a, b in zip(fx.gated_scan_bwd(seqs, x, z, h, small[2]), fx.gated_scan_bwd(seqs, small[0], small[1], h2, small[2])):
        assert torch.equal(a, b)


def test_on_another_stream():
    bounds, jo = _joff([4_000, 3_000])
    seqs = fx.build_sequences(jo)
    x, _ = _draw(71, 7_000, 64, "bf16")
    z, _ = _draw(72, 7_000, 64, "bf16")
    want = fx.gated_scan_fwd(seqs, x, z)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(3):
            got = fx.gated_scan_fwd(seqs, x, z)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_the_same_bits_from_every_call():
    """Many tiles in flight, so that what a tile finds of those before it is never the same twice."""
    n, c = 300_000, 64
    seqs = fx.build_sequences([[0, n]])
    x, _ = _draw(91, n, c, "bf16")
    z, _ = _draw(92, n, c, "bf16", mean=4.0)
    h, last = fx.gated_scan_fwd(seqs, x, z)
    g = fx.gated_scan_bwd(seqs, x, z, h, x)
    for _ in range(10):
        again = fx.gated_scan_fwd(seqs, x, z)
        assert torch.equal(again[0], h) and torch.equal(again[1], last)
        assert all(torch.equal(a, b) for a, b in zip(fx.gated_scan_bwd(seqs, x, z, h, x), g))


def test_sequences_of_a_grid():
    """Every grid of a batch is one sequence of its voxels in index order."""
    from workloads import generators as G
    w = G.workload("sheets_small")
    ijk, jo = w.jagged_ijk()
    g = fx.build_index_grid(torch.from_numpy(ijk).cuda(), jo)
    seqs = fx.build_sequences(g.voxel_joffsets())
    assert seqs.rows == g.num_voxels and seqs.batch_size == g.batch_size
    bounds = np.append(g.voxel_joffsets()[:, 0], g.num_voxels)
    x, rx = _draw(81, g.num_voxels, 8, "f32")
    z, rz = _draw(82, g.num_voxels, 8, "f32")
    h, last = fx.gated_scan_fwd(seqs, x, z)
    ref, rlast, E, El = R.scan(rx, rz, bounds)
    R.check(_f64(h), ref, E, "f32")
    R.check(_f64(last), rlast, El, "f32")


def test_refusals():
    x = torch.zeros((10, 8), device="cuda")
    with pytest.raises(fx.FxError) as e:
        fx.build_sequences([[0, 4], [5, 10]])                 # a gap
    assert e.value.status == -1 and "sequence 1" in str(e.value)
    with pytest.raises(fx.FxError):
        fx.build_sequences([[0, 4], [4, 3]])
    seqs = fx.build_sequences([[0, 10]])
    with pytest.raises(fx.FxError) as e:
        fx.gated_scan_fwd(seqs, x, x.clone(), out=x)          # in place
    assert e.value.status == -1
    with pytest.raises(fx.FxError):
        fx.gated_scan_fwd(seqs, x[:1].expand(10, 8), x)      # rows on top of each other
    with pytest.raises(AssertionError):
        fx.gated_scan_fwd(seqs, x.t().contiguous().t(), x)    # channels apart
    with pytest.raises(AssertionError):
        fx.gated_scan_fwd(seqs, x[:9], x[:9])
    with pytest.raises(AssertionError):
        fx.gated_scan_fwd(seqs, x, x.half())
    with pytest.raises(AssertionError):
        fx.gated_scan_fwd(seqs, x, x.clone(), h0=torch.zeros((2, 8), device="cuda"))
    far = torch.empty(9 * (1 << 26) + 32, dtype=torch.int8, device="cuda").view(torch.float32).as_strided((10, 8), (1 << 24, 1))      # 64 MiB apart
    with pytest.raises(fx.FxError) as e:
        fx.gated_scan_fwd(seqs, far, x)
    assert e.value.status == -5
    # and the call works after the refusals
    assert torch.equal(fx.gated_scan_fwd(seqs, x, x.clone())[0], x)
