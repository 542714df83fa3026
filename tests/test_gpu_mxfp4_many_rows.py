"""MXFP4 of the most rows that one call takes (2^25 - 1), of more than 512
columns: every row as in a short call, bit for bit."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_quantise_and_back():
    from paper_2607_01844_amd import moe
    n, K, P = (1 << 25) - 1, 520, 1 << 16
    g = torch.Generator(device="cuda").manual_seed(5)
    base = torch.randn((P, K), generator=g, device="cuda").bfloat16()
    q, s = moe.moe_mxfp4_quantize(base)
    back = moe.moe_mxfp4_dequantize(q, s, K)
    src = torch.empty((n, K), dtype=torch.bfloat16, device="cuda")
    for part in src.split(P):
        part.copy_(base[:part.shape[0]])
    bq, bs = moe.moe_mxfp4_quantize(src)
    for part in bq.split(P):
        assert torch.equal(part, q[:part.shape[0]])
    for kg in range(bs.shape[0]):
        for part in bs[kg].split(P):
            assert torch.equal(part, s[kg, :part.shape[0]])
    out = moe.moe_mxfp4_dequantize(bq, bs, K, out=src)
    for part in out.split(P):
        assert torch.equal(part, back[:part.shape[0]])
