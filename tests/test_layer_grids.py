"""The launches that a call of many workgroups goes in."""
import ctypes

import numpy as np
import pytest

from paper_2503_22796_amd import binding as B

SLICES = B.lib.difa_testing_slices
SLICES.argtypes = [ctypes.c_int64, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int32]
MOST_THREADS = 512                               # of a workgroup


@pytest.mark.parametrize("workgroups", [0, 1, 7, 2 ** 22 - 1, 2 ** 22, 2 ** 22 + 1, 2 ** 23 + 9, 2 ** 24 - 1, 2 ** 24, 2 ** 24 + 5, 2 ** 31 - 1])
def test_every_workgroup_runs_once_in_launches_below_2_to_32_threads(workgroups):
    first, count = np.zeros(1024, np.int64), np.zeros(1024, np.int64)
    n = SLICES(workgroups, first.ctypes.data, count.ctypes.data, 1024)
    assert n <= 1024 and int(count[:n].sum()) == workgroups
    assert np.array_equal(first[:n], np.cumsum(count[:n]) - count[:n]) and bool((count[:n] > 0).all())
    assert bool((count[:n] * MOST_THREADS < 2 ** 32).all())
    assert bool((first[:n] % 8 == 0).all())       # workgroups stay on their dies
