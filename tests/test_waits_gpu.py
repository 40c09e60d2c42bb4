"""How long a device-side wait lasts that nothing satisfies: the limit that the library's kernels use, by the clock of the host."""
import time

import pytest
import torch

from paper_2502_01703_b200 import binding as B

pytestmark = pytest.mark.gpu


def test_a_wait_with_the_kernels_own_limit_ends_after_seconds():
    B.qless_check()
    x = torch.arange(4096, dtype=torch.float32, device="cuda").view(8, 512)
    before = B.qless_quantize(x, 8)[0]
    torch.cuda.synchronize()
    start = time.perf_counter()
    B.qless_selftest_timeout(0)
    with pytest.raises(B.QlessError) as e:
        B.qless_check()
    took = time.perf_counter() - start
    assert e.value.status == B.ERR_TIMEOUT and "0x1)" in str(e.value)
    assert 1.0 < took < 10.0, took
    B.qless_check()
    assert torch.equal(B.qless_quantize(x, 8)[0], before)
