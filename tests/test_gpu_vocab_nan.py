"""NaN logits reach the losses: of a whole group of 64 columns or of single
ones, in every row or in one (whose neighbours keep their bits)."""
import math

import pytest
import torch

from tests.test_gpu_distill import make

pytestmark = pytest.mark.gpu
SIZES = [(20, 64, 1000, 256), (20, 64, 1003, 64), (300, 72, 999, 1000), (2048, 64, 8192, 4096), (2, 8, 64, 64)]


def losses(x, w, ids, t, vblock):
    from paper_2607_01844_amd import moe
    loss, lse = moe.moe_vocab_loss_fwd(x, w, ids[:, 0].clamp(min=0), vblock)
    dloss, dlse, yk = moe.moe_vocab_distill_fwd(x, w, ids, t, vblock, 0.5)
    return loss, lse, dloss, dlse, yk


@pytest.mark.parametrize("N,H,V,vblock", SIZES)
def test_one_row(N, H, V, vblock):
    x, w, ids, t = make(N, H, V, 4)
    clean = losses(x, w, ids, t, vblock)
    bad = N // 2
    x[bad, 3] = math.nan
    for got, ref in zip(losses(x, w, ids, t, vblock), clean):
        assert got[bad].isnan().all()
        keep = torch.arange(N, device="cuda") != bad
        assert torch.equal(got[keep], ref[keep])


@pytest.mark.parametrize("N,H,V,vblock", SIZES)
@pytest.mark.parametrize("first,many", [(0, 64), (0, 1), (1 << 20, 64), (1 << 20, 1)])
def test_columns(N, H, V, vblock, first, many):
    x, w, ids, t = make(N, H, V, 4)
    ids[0] = -1  # a row without slots
    at = min(first, (V - 1) // 64 * 64)  # the first or the last group
    w[1, at:at + many] = math.nan
    loss, lse, dloss, dlse, _ = losses(x, w, ids, t, vblock)
    assert loss.isnan().all() and lse.isnan().all() and dlse.isnan().all()
    assert dloss[1:].isnan().all() and dloss[0] == 0
