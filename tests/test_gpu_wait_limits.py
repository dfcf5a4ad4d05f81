"""Both forms of a bounded wait, by wall time and by trips, run out at the bound that they are given."""
import time

import pytest

import paper_2606_02823_b200 as qift

pytestmark = pytest.mark.gpu


def test_waits_run_out_at_their_bound():
    qift.qift_selftest_wait_timeout(0, 1)                                             # loads the kernel
    qift.qift_device_status()
    t0 = time.perf_counter()
    qift.qift_selftest_wait_timeout(0, 300_000)
    rc, _ = qift.qift_device_status()
    dt = time.perf_counter() - t0
    assert rc == qift.ERR_TIMEOUT and 0.45 < dt < 1.2                                 # 0.3 s of wall time, then 75 000 trips of 4 us
    assert qift.qift_device_status()[0] == qift.OK
