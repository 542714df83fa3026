"""The distillation reference against its own properties and differences (CPU)."""
import math

import pytest
import torch

from tests import distill_ref as R


def make(N=4, H=8, V=11, K=3, seed=0):
    g = torch.Generator().manual_seed(seed)
    x, w = torch.randn(N, H, generator=g), torch.randn(H, V, generator=g)
    ids = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(N)]).int()
    return x, w, ids, torch.randn(N, K, generator=g)


def test_own_logits_over_the_whole_vocabulary_have_no_loss():
    x, w, _, _ = make(V=6)
    y = x.double() @ w.double()
    ids = torch.arange(6).int().expand(4, 6)
    loss = R.forward(x, w, ids, y, 2.0)[0]
    assert loss.abs().max() < 1e-12
    assert R.logit_grad(x, w, ids, y, torch.ones(4), 2.0).abs().max() < 1e-12


def test_one_slot_is_cross_entropy():
    x, w, ids, t = make(K=1)
    loss, lse, yk = R.forward(x, w, ids, t)
    assert torch.allclose(loss, lse - yk[:, 0])


def test_absent_slots_and_doubled_entries():
    x, w, ids, t = make(K=4)
    ids[0] = -1
    ids[1, 2:] = torch.tensor([11, -5])
    ids[2, 3] = ids[2, 0]
    loss, _, yk = R.forward(x, w, ids, t)
    assert loss[0] == 0 and (yk[0] == 0).all() and (yk[1, 2:] == 0).all()
    short = R.forward(x[1:2], w, ids[1:2, :2], t[1:2, :2])[0]
    assert torch.allclose(loss[1:2], short)
    assert R.logit_grad(x, w, ids, t, torch.ones(4))[0].abs().max() == 0


@pytest.mark.parametrize("tau,absolute", [(1.0, False), (2.5, False), (0.5, True)])
def test_gradient_against_differences(tau, absolute):
    x, w, ids, t = make(seed=3)
    x, w = x.double(), w.double()
    ids[1, 2] = ids[1, 0]
    t[3, 1] = -math.inf
    tlse = torch.logsumexp(t / tau, 1) + 0.3 if absolute else None
    dl = torch.randn(4, generator=torch.Generator().manual_seed(1)).double()
    G = R.logit_grad(x, w, ids, t, dl, tau, tlse)
    h = 1e-6
    for n in range(4):
        for j in range(8):
            up, dn = x.clone(), x.clone()
            up[n, j] += h
            dn[n, j] -= h
            num = ((R.forward(up, w, ids, t, tau, tlse)[0]
                    - R.forward(dn, w, ids, t, tau, tlse)[0]) * dl).sum() / (2 * h)
            assert abs(num - (G @ w.t())[n, j]) < 1e-7
