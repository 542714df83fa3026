"""A teacher's logit of +inf or NaN makes its row's loss and gradient NaN, with
the slots' own sum or with the teacher's log-sum-exp, and no other row's."""
import math

import pytest
import torch

from tests.test_gpu_distill import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("absolute", [False, True])
@pytest.mark.parametrize("value", [math.inf, math.nan])
@pytest.mark.parametrize("K,slot", [(4, 2), (130, 129), (1, 0)])
def test_row_becomes_nan(absolute, value, K, slot):
    from paper_2607_01844_amd import moe
    x, w, ids, t = make(12, 16, 90, K)
    tlse = torch.logsumexp(t, 1) + 0.5 if absolute else None
    dl = torch.ones(12, device="cuda")
    clean = moe.moe_vocab_distill_fwd(x, w, ids, t, 32, 2.0, tlse)
    cdx, _ = moe.moe_vocab_distill_bwd(x, w, ids, t, clean[1], clean[2], dl, 32, 2.0, tlse)
    t[3, slot] = value
    loss, lse, yk = moe.moe_vocab_distill_fwd(x, w, ids, t, 32, 2.0, tlse)
    dx, dw = moe.moe_vocab_distill_bwd(x, w, ids, t, lse, yk, dl, 32, 2.0, tlse)
    assert loss[3].isnan() and dx[3].isnan().all() and dw.isnan().all()
    ok = torch.arange(12, device="cuda") != 3
    assert torch.equal(loss[ok], clean[0][ok]) and torch.equal(dx[ok], cdx[ok])
    ids[3, slot] = -1  # an absent slot's may be anything
    loss, lse, yk = moe.moe_vocab_distill_fwd(x, w, ids, t, 32, 2.0, tlse)
    assert loss[3].isfinite()
