"""Copies of W and sums of dx of more than the 2^27 elements that one grid of
their kernels covers (they step over the rest)."""
import pytest

from tests.test_gpu_distill import check, make

pytestmark = pytest.mark.gpu


def test_copy_of_many_columns():
    N, H, V = 3, 4096, 33001
    assert H * V > 1 << 27 and V % 8
    check(*make(N, H, V, 2), 1 << 16)


def test_sum_of_many_rows():
    N, H, V = 16387, 8200, 64
    assert N * H > 1 << 27
    check(*make(N, H, V, 3), 64)
