"""Gradients of distillation with few rows: the logit gradients are held in two
bf16 parts, so dx and dw carry one rounding to bf16 and little beside it.

Tolerances (U = 2^-24): those of test_gpu_distill.py, with 2^-16 of an entry of
the logit gradients (the second part is off by 2^-8 of the first's rounding, at
most 2^-8) in place of 2^-8, and sums of twice the terms."""
import pytest
import torch

from tests import distill_ref as R
from tests.test_gpu_distill import make

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def check(x, w, ids, t, vblock, tau=1.0, tlse=None, seed=1):
    from paper_2607_01844_amd import moe
    N, H = x.shape
    V, K = w.shape[1], ids.shape[1]
    dl = torch.randn(N, generator=torch.Generator().manual_seed(seed)).to("cuda")
    _, lse, yk = moe.moe_vocab_distill_fwd(x, w, ids, t, vblock, tau, tlse)
    dx, dw = moe.moe_vocab_distill_bwd(x, w, ids, t, lse, yk, dl, vblock, tau, tlse)
    cx, cw, cids, ct, ctl, cdl = [None if a is None else a.cpu() for a in (x, w, ids, t, tlse, dl)]
    _, rlse, _ = R.forward(cx, cw, cids, ct, tau, ctl)
    p, _ = R.teacher(cids, ct, V, tau, ctl)
    ey = H * U * (cx.double().abs() @ cw.double().abs()).amax(1)
    tt = torch.where(p > 0, (ct.double() / tau).abs(), 0.0).amax(1)
    ep = (100 + 4 * tt + (0 if ctl is None else 2 * ctl.double().abs())) * U
    el = ey / tau + 200 * U + 2 * U * rlse.abs()
    G = R.logit_grad(cx, cw, cids, ct, cdl, tau, ctl)
    f = cdl.double().abs()[:, None] / tau
    q = torch.softmax(cx.double() @ cw.double() / tau, 1)
    eG = f * (p.sum(1)[:, None] * q * (ep + 2 * el + ey / tau + 40 * U)[:, None])
    there = (cids >= 0) & (cids < V)
    eG.scatter_add_(1, torch.where(there, cids, 0).long(), f * p * (ep[:, None] + K * U))
    eG += 2.0 ** -16 * G.abs() + 2.0 ** -133
    ex = eG @ cw.double().abs().t() + 2 * V * U * (G.abs() @ cw.double().abs().t())
    ew = cx.double().abs().t() @ eG + 2 * N * U * (cx.double().abs().t() @ G.abs())
    rx, rw = G @ cw.double().t(), cx.double().t() @ G
    assert ((dx.cpu().double() - rx).abs() <= ex + 2.0 ** -8 * (rx.abs() + ex) + 2.0 ** -133).all()
    assert ((dw.cpu().double() - rw).abs() <= ew + 2.0 ** -8 * (rw.abs() + ew) + 2.0 ** -133).all()


SIZES = [(1, 64, 1000, 4, 256), (1, 8, 1, 1, 8), (2, 264, 4099, 32, 1 << 20), (3, 520, 1003, 7, 200),
         (16, 128, 2000, 32, 512), (31, 72, 777, 5, 64), (64, 136, 3001, 64, 1024), (64, 64, 20000, 3, 4096),
         (33, 2048, 1024, 200, 1024), (5, 16, 300, 130, 128)]


@pytest.mark.parametrize("N,H,V,K,vblock", SIZES)
@pytest.mark.parametrize("tau,absolute", [(1.0, False), (0.5, True)])
def test_one_rounding(N, H, V, K, vblock, tau, absolute):
    x, w, ids, t = make(N, H, V, K, seed=N)
    tlse = torch.logsumexp(t / tau, 1) + 0.25 if absolute else None
    check(x, w, ids, t, vblock, tau, tlse)


def test_repeated_and_absent_slots():
    x, w, ids, t = make(20, 32, 300, 13)
    ids[:, :5] = 77
    ids[::3, 5:] = -1
    ids[7] = 300
    check(x, w, ids, t, 128)


def test_largest_tile():
    """Columns enough for the 256-row tile."""
    check(*make(64, 64, 70000, 9), 1 << 20)
