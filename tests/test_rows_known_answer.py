"""Dropout's generator against the known answer that its authors publish with it: Philox4x32 with seven rounds at zero counter and
key."""
import numpy as np

import rows_reference as R

WORDS = (0x5F6FB709, 0x0D893F64, 0x4F121F81, 0x4F730A48)


def test_zero_counter_and_key():
    halves = [h for w in WORDS for h in (w & 0xFFFF, w >> 16)]
    for e, v in enumerate(halves):          # number v is kept at t = v and dropped from t = v + 1 on
        kept = [R.keep_mask(1, 8, t / 65536, 0, 0)[0, e] for t in (v, v + 1)]
        assert kept == [True, False], (e, v)
    assert np.array_equal(R.keep_mask(1, 8, 0.5, 0, 0)[0], np.array(halves) >= 32768)
