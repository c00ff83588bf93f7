"""Calls of 8-bit products that are checked whole before anything is enqueued (no GPU: dry-run mode)."""
import ctypes as C

import pytest

FAKE = 0x10000   # a non-NULL, 256-byte aligned address; never dereferenced in dry-run mode


@pytest.fixture(scope="module")
def mq():
    from paper_2508_09204_amd import binding
    binding.moqe_set_dry_run(True)
    yield binding
    binding.moqe_set_dry_run(False)


@pytest.mark.parametrize("M,n,code", [(1 << 20, 1 << 16, 0), (1 << 24, 1 << 24, -2), (1 << 23, 1 << 22, -2), (33, 1 << 24, 0)])
@pytest.mark.parametrize("flags", [0, 8])
def test_launches_past_the_limit_are_refused_with_the_arguments(mq, M, n, code, flags):
    a, mat = mq._F8Rows(FAKE, FAKE, 128, 4), (mq._F8Mat * 1)(mq._F8Mat(FAKE, n, 100, 0))
    y = mq._F8Result(FAKE, n, 0, mq._F8Rows())
    assert mq.lib.moqe_f8_gemm(C.byref(a), None, None, M, 1, mat, 1, C.byref(y), flags, None, 0, None) == code
