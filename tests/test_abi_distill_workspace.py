"""The distillation workspace stays that of the caller's block: beside
moe_vocab_loss's and the teacher's data, what taking blocks together may add is
bounded, with a copy of W's columns (V no multiple of 8) or without."""
import ctypes

import pytest

MIB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    from paper_2607_01844_amd import moe
    return moe.lib


def sizes(lib, N, H, V, vblock, K):
    n, v = ctypes.c_size_t(), ctypes.c_size_t()
    assert lib.moe_vocab_distill_workspace_bytes(N, H, V, vblock, K, ctypes.byref(n)) == 0
    assert lib.moe_vocab_loss_workspace_bytes(N, H, V, vblock, ctypes.byref(v)) == 0
    vb = min(vblock, V)
    teacher = 4 * N * (3 * K + 8) + 4 * N * (vb // 2048 + 2) + 4096
    return n.value - v.value - teacher


@pytest.mark.parametrize("N,H,V,vblock,K", [
    (2, 8192, 200001, 4096, 64), (128, 7168, 151669, 2048, 64), (1, 262144, 100003, 64, 1),
    (2, 2632, 76658, 4096, 8)])
def test_few_rows_do_not_take_a_copy_of_w(lib, N, H, V, vblock, K):
    # the copy of blocks taken together; G and partial sums of so few rows
    few = 256 * MIB + 2 * N * V + 170 * 4 * N * H
    assert sizes(lib, N, H, V, vblock, K) <= min(few, 448 * MIB)


def test_bounded_over_the_range(lib):
    for N in (1, 2, 7, 64, 128, 500, 1000, 4096, 32768, 1 << 20):
        for H in (8, 64, 520, 2048, 7168, 16384, 262144):
            for V in (1000, 32003, 76658, 200000, 200001, 5_000_000, 34_000_003):
                for vblock in (8, 64, 512, 4096, 16384, 1 << 19):
                    assert sizes(lib, N, H, V, vblock, 64) <= 448 * MIB, (N, H, V, vblock)
