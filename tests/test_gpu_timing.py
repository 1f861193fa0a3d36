"""Events of the per-kernel timing: a read takes all that has been recorded, whichever of the two reads it is."""
import ctypes

import pytest
import torch

from paper_2505_07004_b200 import api as libgq

pytestmark = pytest.mark.gpu


def read(count):
    ms, cnt = (ctypes.c_double * 17)(*[-1.0] * 17), (ctypes.c_uint64 * 17)(*[99] * 17)
    L = libgq.lib()
    assert (L.gq_kernel_timing_read(ms, cnt) if count is None else L.gq_kernel_timing_read_all(ms, cnt, count)) == 0
    return list(ms), list(cnt)


@pytest.mark.parametrize("count", [None, 1, 14, 15])
def test_a_read_discards_what_it_does_not_report(count):
    x = torch.randn(3, 100, device="cuda:0")
    read(17)
    libgq.lib().gq_kernel_timing_enable(1)
    try:
        for _ in range(3):
            libgq.gq_token_logprobs(x)
    finally:
        libgq.lib().gq_kernel_timing_enable(0)
    ms, cnt = read(count)
    reported = 14 if count is None else count
    assert cnt[reported:] == [99] * (17 - reported) and ms[reported:] == [-1.0] * (17 - reported)
    assert cnt[:reported] == [0] * 14 + [3] if count == 15 else cnt[:reported] == [0] * reported
    assert read(17)[1] == [0] * 17
