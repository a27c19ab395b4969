"""LDS of the step's kernels: what they declare and the used bits of the largest worker, 65536 bytes at most (from the compiler's report of the last build)."""
import os

import pytest

from tests.test_kernel_residency import REPORT

USED_BITS = 262144 // 8  # BR_KV_MAX_BLOCKS


def _lines():
    return [line for line in open(REPORT) if line.startswith("_Z12br_kv_k_stepI")] if os.path.exists(REPORT) else []


@pytest.mark.skipif(not os.path.exists(REPORT), reason="no build report")
def test_the_largest_worker_fits():
    lines = _lines()
    assert len(lines) == 12  # rows to a thread: 1, 2, 4; with and without the token list; blocks with one holder or several
    for line in lines:
        assert int(line.split("lds=")[1].split()[0]) + USED_BITS <= 65536, line.strip()
