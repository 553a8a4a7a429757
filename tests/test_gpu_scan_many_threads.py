"""More rows than one launch has threads for."""
import pytest
import torch

import paper_2407_01781_amd as fx

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
