"""Sizes of the join's workspace at the ends of what it takes."""
import ctypes

import pytest

from paper_2010_04902_b200 import binding as bz
from paper_2010_04902_b200 import build as bz_build


@pytest.fixture(scope="module")
def L():
    bz_build.build()
    return bz.lib()


@pytest.mark.parametrize("m", [0, 1, 4, 777, (1 << 31) - 1])
def test_no_columns(L, m):
    """A division by the threads that no column needs ended the process."""
    for groups in (0, 1, m):
        if groups <= 1 or m:
            assert L.bz_join_workspace_bytes(m, 0, groups) == 256


def test_no_columns_in_a_call(L):
    F = ctypes.c_void_p(256)      # never dereferenced
    n0 = bz.kernel_launch_count()
    assert L.bz_join_backward(F, 0, F, 0, bz.F32, 4, 0, bz.NORM_RMS, F, F, 2, 1.0, 1.0, 0.0, None, F, F, F, 0, F, 0, F, 0, F, 0, F, F, F, None, 0, None) == bz.OK
    assert bz.kernel_launch_count() == n0


def test_the_smallest_and_the_widest(L):
    for m in (0, 1, 2, 15, 16, 4097, 1 << 20):
        for n in (1, 31, 32, 33, 511, 512, 513, 682, 684, 4096, 4097, 8192, 8193, bz.MAX_WIDTH):
            for groups in {0, 1, m}:
                size = L.bz_join_workspace_bytes(m, n, groups)
                assert size >= 256 and size % 256 == 0 and size >= 2 * 4 * n
