"""Integer products of few rows whose long contractions stay whole: 32x32 tiles on four and on six stages, whole and ragged last k-tiles."""

import pytest

import test_gpu_integers as base

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k", [(8, 8200, 8192), (5, 8225, 8200), (20, 16384, 8193), (32, 8209, 7700), (31, 8193, 7807), (17, 9000, 20001), (8, 8200, 8320), (6, 16384, 7681)])
def test_sums_are_exact(m, n, k):
    base.test_sums_are_exact(m, n, k)
