"""Quantisation along the columns of many matrices, whose rows together pass
2^25 (a result has B C rows): each matrix as by itself, bit for bit."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_long_columns():
    from paper_2607_01844_amd import moe
    B, R, C = 1025, 1 << 15, 8
    g = torch.Generator(device="cuda").manual_seed(7)
    src = torch.randn((B, R, C), generator=g, device="cuda").bfloat16()
    q, s = moe.moe_mxfp4_quantize(src, transpose=True)
    for b in (0, 1, 511, 1023, 1024):
        q1, s1 = moe.moe_mxfp4_quantize(src[b].clone(), transpose=True)
        assert torch.equal(q[b], q1) and torch.equal(s[b], s1)
        rows = moe.moe_mxfp4_quantize(src[b].t().contiguous())
        assert torch.equal(q1, rows[0]) and torch.equal(s1, rows[1])
