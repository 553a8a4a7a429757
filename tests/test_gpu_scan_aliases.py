"""The recurrence refuses outputs that lie where it still reads: states in and out in one table, one table for two gradients.
Nothing is launched for a refused call."""
import pytest
import torch

import paper_2407_01781_amd as fx
from paper_2407_01781_amd import binding as B

pytestmark = pytest.mark.gpu
N, C = 40, 66                   # two slabs, the second of two channels: its lanes take the last two of the first along


@pytest.fixture
def data():
    rows = [torch.full((N, C), 1.0, device="cuda") for _ in range(6)]
    states = [torch.full((2 * 3 * C,), 2.0, device="cuda") for _ in range(3)]
    return fx.build_sequences([[0, 10], [10, 10], [10, N]]), rows, states


def _refused(status, word):
    assert status == -1 and word in B.lib.fx_last_error().decode()


def test_forward(data):
    seqs, (x, z, h, *_), (t, u, _) = data
    call = lambda h0, last: B.lib.fx_gated_scan_fwd(seqs._h, x.data_ptr(), C, z.data_ptr(), C, 0, C, 0, h0, h.data_ptr(), C, last, None)
    p, size = t.data_ptr(), 4 * 3 * C
    for h0, last in ((p, p), (p, p + 4), (p + size - 4, p)):
        _refused(call(h0, last), "d_last")
    assert bool((h == 1).all()) and bool((t == 2).all())
    torch.cuda.synchronize()
    assert call(p, p + size) == 0 and call(None, u.data_ptr()) == 0 and call(p, None) == 0      # side by side, and one alone
    torch.cuda.synchronize()


def test_backward(data):
    seqs, (x, z, h, gh, gx, gz), (t, u, w) = data
    call = lambda gx, gz, h0, gl, g0: B.lib.fx_gated_scan_bwd(seqs._h, x.data_ptr(), C, z.data_ptr(), C, h.data_ptr(), C, gh.data_ptr(), C, 0, C, 0, h0, gl,
                                                              gx.data_ptr(), C, gz.data_ptr(), C, g0, None)
    p, q, r, size = t.data_ptr(), u.data_ptr(), w.data_ptr(), 4 * 3 * C
    _refused(call(gx, gx, p, q, r), "d_gx and d_ggate")
    for h0, gl, g0 in ((p, q, p), (p, q, q), (None, q, q + size - 4), (p + 4, None, p)):
        _refused(call(gx, gz, h0, gl, g0), "d_gh0")
    assert bool((gx == 1).all()) and bool((gz == 1).all()) and all(bool((v == 2).all()) for v in (t, u, w))
    torch.cuda.synchronize()
    assert call(gx, gz, p, q, r) == 0 and call(gx, gz, p, p, r) == 0 and call(gx, gz, p, None, p + size) == 0     # inputs may be one table
    torch.cuda.synchronize()
