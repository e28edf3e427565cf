"""The device-side wait of the tensor-core product where it runs out: a bounded wait of the debug build, for something that nothing does."""
import ctypes
import os
import time

import pytest

import paper_2604_00529_b200 as mxq

from test_debug_build import LIB

TIMEOUT = -8


def test_release_build_has_no_test_wait():
    lanes = ctypes.c_uint(7)
    assert mxq.load_library().mxq_debug_wait(ctypes.c_uint(1), ctypes.byref(lanes)) == 0 and lanes.value == 7


@pytest.mark.gpu
def test_a_wait_that_runs_out_ends_for_the_whole_warp_and_is_reported():
    if not os.path.exists(LIB):
        pytest.fail("libmxq_debug.so is not built: python -m paper_2604_00529_b200.build --debug")
    D = ctypes.CDLL(LIB)
    D.mxq_debug_wait.argtypes = [ctypes.c_uint, ctypes.POINTER(ctypes.c_uint)]
    assert D.mxq_debug_wait(1001, ctypes.byref(ctypes.c_uint())) == -4 and D.mxq_debug_wait(1, None) == -1
    assert D.mxq_wait_status(1) == 0
    for ms in (1, 50):
        lanes = ctypes.c_uint(0xFFFFFFFF)
        began = time.monotonic()
        assert D.mxq_debug_wait(ms, ctypes.byref(lanes)) == 1
        took = time.monotonic() - began
        print("a wait of %d ms took %.1f ms" % (ms, 1e3 * took))
        assert lanes.value == 0                              # no lane goes on without the others
        assert ms * 1e-3 <= took < 5
        assert D.mxq_wait_status(0) == TIMEOUT               # remembered until it is reset
        assert D.mxq_wait_status(1) == TIMEOUT
        assert D.mxq_wait_status(0) == 0
    assert mxq.load_library().mxq_wait_status(0) == 0       # (the other library's kernels)
