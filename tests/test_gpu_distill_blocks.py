"""Distillation of few rows whose blocks go through a copy of W's columns, where
only some of the caller's blocks are taken together (256 MiB of the copy)."""
import pytest

from tests.test_gpu_distill import check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,H,V,K,vblock", [(2, 8192, 20001, 9, 1024), (40, 6144, 30003, 5, 4096),
                                            (5, 16384, 9001, 3, 64)])
def test_copies_of_some_blocks(N, H, V, K, vblock):
    check(*make(N, H, V, K, seed=H), vblock)
