"""With transpose the rows of the result are the columns of the source: limits
are those of them (B C < 2^25, R a dimension), not of the source's rows."""
import pytest

from tests.abi_cases import P, Z


@pytest.fixture(scope="module")
def lib():
    import torch
    if torch.cuda.is_available():
        pytest.skip("dummy pointers are only safe without a GPU")
    from paper_2607_01844_amd import moe
    return moe.lib


def quant(lib, B, R, C, transpose=1, p=P):
    return lib.moe_mxfp4_quantize(p, B, R, C, transpose, p, p, Z)


@pytest.mark.parametrize("B,R,C", [(1024, 1 << 15, 8), (65535, 262144, 8), (1, 262144, 262144), (128, 262144, 4096)])
def test_within_the_limits(lib, B, R, C):
    assert quant(lib, B, R, C) != -1  # (no device here: the launch itself fails)
    assert quant(lib, B, R, C, p=Z) == -1 and b"NULL" in lib.moe_last_error()


@pytest.mark.parametrize("B,R,C", [(128, 64, 262144), (65536, 8, 8), (-1, 8, 8), (2, -8, 8), (2, 12, 8),
                                   (2, 8, 12), (2, 262152, 8), (2, 1 << 40, 8), (1 << 40, 8, 8), (2, 8, 262152)])
def test_beyond_them(lib, B, R, C):
    assert quant(lib, B, R, C) == -1


def test_nothing_to_do(lib):
    assert quant(lib, 0, 60, 8, p=Z) == quant(lib, 5, 0, 8, p=Z) == 0
