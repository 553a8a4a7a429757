"""More rows than one launch has threads for."""
import pytest
import torch

import paper_2407_01781_amd as fx
from paper_2407_01781_amd import binding as B

pytestmark = pytest.mark.gpu


def test_steps_of_more_rows_than_threads():
    n = (1 << 32) + 1_000                   # 43 GB of rows of one channel
    x = torch.zeros((n, 1), dtype=torch.bfloat16, device="cuda")
    s = torch.full((n, 1), 2.0, device="cuda")
    ends = (0, 1, (1 << 32) - 300, (1 << 32) - 257, (1 << 32) - 256, (1 << 32) - 1, 1 << 32, n - 1)
    for i, r in enumerate(ends):
        s[r] = i + 3.0
    h, new = fx.gated_scan_step(x, x, s, new_state=s)
    assert new is s
    for i, r in enumerate(ends):            # half of the state: sigmoid(0) = 1/2, exactly
        assert float(h[r]) == float(s[r]) == (i + 3.0) / 2
        h[r] = s[r] = 1.0
    part = 1 << 28                          # comparisons of a part at a time: torch's own kernels count in 32 bits too
    assert all(bool((t[a:a + part] == 1).all()) for t in (h, s) for a in range(0, n, part))


def test_more_tiles_than_threads():
    """Refused on the host: of 2^31 - 1 rows of 129 channels nothing but the sequences' table is there."""
    n, c = (1 << 31) - 1, 129
    seqs = fx.build_sequences([[0, n]])
    x = torch.empty(1, dtype=torch.bfloat16, device="cuda")
    p = [x.data_ptr() + (i << 43) for i in range(3)]
    assert B.lib.fx_gated_scan_fwd(seqs._h, p[0], c, p[1], c, 2, c, 0, None, p[2], c, None, None) == -5
    assert b"too many tiles" in B.lib.fx_last_error()
