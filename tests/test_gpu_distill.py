"""Distillation from a teacher's top logits on the GPU against the dense 64-bit
reference.

Tolerances (U = 2^-24).  A logit is an fp32 sum of H exact products: off by at
most ey = H U sum |x w|.  lse moves by ey / tau at most, and its own sum of
exponentials (relative error of one: 2^-22 + 20 U for an argument within 20 of
the maximum; the sums add 64 + log2 terms) by 200 U; its fp32 value by U |lse|.
p is good to 100 U + the rounding of t / tau (|t / tau| U).  G is rounded to
bf16 (2^-8 of itself), dx and dw once more, and their fp32 sums carry (terms) U."""
import math

import pytest
import torch

from tests import distill_ref as R

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def make(N, H, V, K, seed=0, device="cuda"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(N, H, generator=g).bfloat16()
    w = (torch.randn(H, V, generator=g) * 0.1).bfloat16()
    ids = (torch.rand(N, K, generator=g) * V).int()  # entries may repeat
    t = torch.randn(N, K, generator=g) * 2
    return [a.to(device) for a in (x, w, ids, t)]


def check(x, w, ids, t, vblock, tau=1.0, tlse=None, seed=1):
    from paper_2607_01844_amd import moe
    N, H = x.shape
    V, K = w.shape[1], ids.shape[1]
    dl = torch.randn(N, generator=torch.Generator().manual_seed(seed)).to("cuda")
    loss, lse, yk = moe.moe_vocab_distill_fwd(x, w, ids, t, vblock, tau, tlse)
    dx, dw = moe.moe_vocab_distill_bwd(x, w, ids, t, lse, yk, dl, vblock, tau, tlse)
    torch.cuda.synchronize()
    c = [None if a is None else a.cpu() for a in (x, w, ids, t, tlse, dl)]
    cx, cw, cids, ct, ctl, cdl = c
    rloss, rlse, ryk = R.forward(cx, cw, cids, ct, tau, ctl)
    p, logp = R.teacher(cids, ct, V, tau, ctl)
    P = p.sum(1)
    mag = cx.double().abs() @ cw.double().abs()
    ey = H * U * mag.amax(1)
    tt = torch.where(p > 0, (ct.double() / tau).abs(), 0.0).amax(1)
    ep = (100 + 4 * tt + (0 if ctl is None else 2 * ctl.double().abs())) * U
    el = ey / tau + 200 * U + 2 * U * rlse.abs()
    assert ((yk.cpu().double() - ryk).abs() <= ey[:, None]).all()
    assert ((lse.cpu().double() - rlse).abs() <= el).all()
    big = torch.where(p > 0, (logp - ryk / tau + rlse[:, None]).abs(), 0.0)
    eloss = (p * (ep[:, None] * (1 + big) + (el + ey / tau)[:, None]
                  + 4 * U * (ryk.abs() / tau + rlse.abs()[:, None] + logp.abs()))).sum(1)
    assert ((loss.cpu().double() - rloss).abs() <= eloss + K * U * (p * big).sum(1)).all()
    G = R.logit_grad(cx, cw, cids, ct, cdl, tau, ctl)
    f = cdl.double().abs()[:, None] / tau
    q = torch.softmax(cx.double() @ cw.double() / tau, 1)
    eG = f * (P[:, None] * q * (ep + 2 * el + ey / tau + 40 * U)[:, None])
    there = (cids >= 0) & (cids < V)
    eG.scatter_add_(1, torch.where(there, cids, 0).long(), f * p * (ep[:, None] + K * U))
    eG += 2.0 ** -8 * G.abs() + 2.0 ** -133
    ex = eG @ cw.double().abs().t() + V * U * (G.abs() @ cw.double().abs().t())
    ew = cx.double().abs().t() @ eG + N * U * (cx.double().abs().t() @ G.abs())
    rx, rw = G @ cw.double().t(), cx.double().t() @ G
    assert ((dx.cpu().double() - rx).abs() <= ex + 2.0 ** -8 * (rx.abs() + ex) + 2.0 ** -133).all()
    assert ((dw.cpu().double() - rw).abs() <= ew + 2.0 ** -8 * (rw.abs() + ew) + 2.0 ** -133).all()
    return loss, lse, yk, dx, dw


SIZES = [(1, 8, 1, 1, 8), (3, 8, 5, 2, 8), (65, 64, 100, 7, 64), (256, 128, 1000, 8, 256),
         (130, 72, 777, 33, 200), (40, 40, 4099, 256, 1024), (300, 264, 3001, 5, 8),
         (129, 136, 2600, 64, 4096), (2, 520, 70001, 100, 1 << 20)]


@pytest.mark.parametrize("N,H,V,K,vblock", SIZES)
@pytest.mark.parametrize("tau,absolute", [(1.0, False), (2.0, True)])
def test_sizes(N, H, V, K, vblock, tau, absolute):
    x, w, ids, t = make(N, H, V, K, seed=N)
    tlse = torch.logsumexp(t / tau, 1) + 0.25 if absolute else None
    check(x, w, ids, t, vblock, tau, tlse)


def test_large_tile():
    """Enough tiles for the 256-row tile in both directions."""
    check(*make(2048, 64, 8192, 20), 8192)
    check(*make(2048, 64, 8200, 3), 4096, 0.7)


def test_slots_on_the_edges_of_groups_and_blocks():
    x, w, ids, t = make(70, 64, 1000, 16)
    edges = torch.tensor([0, 63, 64, 127, 128, 191, 199, 200, 201, 255, 256, 511, 512, 998, 999, 600])
    ids[:] = edges[None].int()
    for vb in (64, 200, 256, 1000):
        check(x, w, ids, t, vb)


def test_all_rows_share_one_group():
    x, w, ids, t = make(260, 32, 640, 64)
    ids[:] = torch.arange(64).int()[None] + 128
    check(x, w, ids, t, 640)


def test_same_entry_in_every_slot():
    x, w, ids, t = make(20, 32, 300, 130)
    ids[:] = 77
    check(x, w, ids, t, 128)


def test_absent_slots_and_empty_rows():
    x, w, ids, t = make(100, 48, 500, 9)
    ids[::3] = -1
    ids[1::3, 4:] = 500  # beyond the vocabulary
    ids[2::3, 0] = -(1 << 31)
    t[4, :] = -math.inf  # a teacher that gives nothing
    t[5, 1] = torch.finfo(torch.float32).min
    loss, lse, yk, dx, dw = check(x, w, ids, t, 128)
    assert (loss[::3] == 0).all() and (dx[::3] == 0).all() and (yk[::3] == 0).all()
    assert loss[4] == 0 and (dx[4] == 0).all()
    # logits of absent slots may hold anything
    t2 = t.clone()
    t2[ids < 0] = math.nan
    t2[ids >= 500] = math.inf
    again = check(x, w, ids, t2, 128)
    for a, b in zip((loss, lse, yk, dx, dw), again):
        assert torch.equal(a, b)


def test_nan_of_one_teacher_row_stays_there():
    from paper_2607_01844_amd import moe
    x, w, ids, t = make(12, 16, 90, 4)
    t[3, 2] = math.nan
    loss, lse, yk = moe.moe_vocab_distill_fwd(x, w, ids, t, 32)
    dl = torch.ones(12, device="cuda")
    dx, _ = moe.moe_vocab_distill_bwd(x, w, ids, t, lse, yk, dl, 32)
    ok = torch.arange(12, device="cuda") != 3
    assert torch.isnan(loss[3]) and torch.isfinite(loss[ok]).all()
    assert torch.isnan(dx[3]).all() and torch.isfinite(dx[ok]).all()


def test_no_rows():
    from paper_2607_01844_amd import moe
    x, w, ids, t = make(0, 16, 90, 4)
    loss, lse, yk = moe.moe_vocab_distill_fwd(x, w, ids, t, 32)
    dw = torch.full((16, 90), 3.0, dtype=torch.bfloat16, device="cuda")
    moe.moe_vocab_distill_bwd(x, w, ids, t, lse, yk, loss, 32, dw_voc=dw)
    assert loss.numel() == 0 and (dw == 0).all()


def test_one_slot_is_the_plain_loss():
    """A teacher of one slot a row is the target of moe_vocab_loss."""
    from paper_2607_01844_amd import moe
    x, w, ids, t = make(200, 64, 1000, 1)
    loss, lse, yk = moe.moe_vocab_distill_fwd(x, w, ids, t, 256)
    want, wlse = moe.moe_vocab_loss_fwd(x, w, ids[:, 0].contiguous(), 256)
    assert torch.equal(lse, wlse)
    assert (loss + want).abs().max() <= 4 * U * lse.abs().max()


def test_same_bits_at_any_workspace_and_on_another_stream():
    from paper_2607_01844_amd import moe
    x, w, ids, t = make(500, 64, 3000, 12)
    dl = torch.ones(500, device="cuda")

    def both():
        loss, lse, yk = moe.moe_vocab_distill_fwd(x, w, ids, t, 512, 1.5)
        return (loss, lse, yk, *moe.moe_vocab_distill_bwd(x, w, ids, t, lse, yk, dl, 512, 1.5))

    a = both()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = both()
    torch.cuda.current_stream().wait_stream(s)
    for u, v in zip(a, b):
        assert torch.equal(u, v)
    # a workspace for the forward alone: its blocks go one by one
    n = 4 * 500 * (2 * 8 + 3 + 12 + 12 + 1) + 8 * 256
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    loss, lse, yk = (torch.empty_like(v) for v in a[:3])
    st = torch.cuda.current_stream().cuda_stream
    assert moe.lib.moe_vocab_distill_fwd(
        x.data_ptr(), w.data_ptr(), ids.data_ptr(), t.data_ptr(), None, 1.5, 500, 64, 3000, 512, 12,
        loss.data_ptr(), lse.data_ptr(), yk.data_ptr(), ws.data_ptr(), n, st) == 0
    torch.cuda.synchronize()
    for u, v in zip(a, (loss, lse, yk)):
        assert torch.equal(u, v)


def test_graph_replays():
    from paper_2607_01844_amd import moe
    x, w, ids, t = make(300, 64, 2000, 10)
    dl = torch.ones(300, device="cuda")

    def both():
        loss, lse, yk = moe.moe_vocab_distill_fwd(x, w, ids, t, 512)
        return (loss, lse, yk, *moe.moe_vocab_distill_bwd(x, w, ids, t, lse, yk, dl, 512))

    want = [v.clone() for v in both()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = both()
    for _ in range(3):
        for v in out:
            v.fill_(math.nan)
        g.replay()
        torch.cuda.synchronize()
        for u, v in zip(out, want):
            assert torch.equal(u, v)
        for u, v in zip(both(), want):
            assert torch.equal(u, v)


def test_binding_refuses():
    from paper_2607_01844_amd import moe
    x, w, ids, t = make(10, 16, 90, 4)
    for call, err in [
            (lambda: moe.moe_vocab_distill_fwd(x.float(), w, ids, t, 32), TypeError),
            (lambda: moe.moe_vocab_distill_fwd(x, w[:8], ids, t, 32), ValueError),
            (lambda: moe.moe_vocab_distill_fwd(x, w, ids[:9], t, 32), ValueError),
            (lambda: moe.moe_vocab_distill_fwd(x, w, ids, t[:, :3], 32), ValueError),
            (lambda: moe.moe_vocab_distill_fwd(x, w, ids.long(), t, 32), TypeError),
            (lambda: moe.moe_vocab_distill_fwd(x, w, ids, t, 32, 1.0, t[:, 0]), ValueError),
            (lambda: moe.moe_vocab_distill_fwd(x, w, ids, t, 32, 0.0), moe.MoEError),
            (lambda: moe.moe_vocab_distill_fwd(x, w, ids, t, 30), moe.MoEError),
            (lambda: moe.moe_vocab_distill_fwd(x, w, ids[:, :0], t[:, :0], 32), moe.MoEError)]:
        with pytest.raises(err):
            call()
