"""Arguments of the 4-bit cache's calls that the library takes or refuses before
any launch (no GPU)."""
import pytest

import paper_2606_24467_gb300 as ckv


def test_stall_hook_limits():
    for bad in (-1, 99_999, 2_000_000_001):
        with pytest.raises(ckv.CompressKVError):
            ckv.debug_stall_next_q4_attend(bad)
    ckv.debug_stall_next_q4_attend(1_000_000)
    ckv.debug_stall_next_q4_attend(0)  # cancelled: no later call stalls
