"""Backward of both vocabulary losses without rows: dw is exact zeros up to its
last element, from one column to more than 2^32 elements."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,V", [(8, 1), (16, 90), (24, 1031), (16384, (1 << 18) + 1)])
def test_zeros(H, V):
    from paper_2607_01844_amd import moe
    dev = dict(device="cuda")
    x = torch.empty((0, H), dtype=torch.bfloat16, **dev)
    w = torch.empty((H, V), dtype=torch.bfloat16, **dev)
    f, i = torch.empty(0, **dev), torch.empty(0, dtype=torch.int32, **dev)
    ids, t = torch.empty((0, 4), dtype=torch.int32, **dev), torch.empty((0, 4), **dev)
    buf = torch.empty(H * V + 64, dtype=torch.bfloat16, **dev)
    dw = buf[:H * V].view(H, V)
    for call in (lambda: moe.moe_vocab_loss_bwd(x, w, i, f, f, 4096, dw_voc=dw),
                 lambda: moe.moe_vocab_distill_bwd(x, w, ids, t, f, t, f, 4096, dw_voc=dw)):
        buf.fill_(3)
        dx, out = call()
        assert out is dw and dx.shape == (0, H)
        for part in buf[:H * V].split(1 << 30):
            assert not part.any()
        assert (buf[H * V:] == 3).all()
